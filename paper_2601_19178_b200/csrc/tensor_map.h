// Tensor maps: rows of 16-bit elements in device memory, fetched in boxes of whole or part rows.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

namespace ckv {

// A tensor of 16-bit elements.  false if the driver cannot encode it.
inline bool encode_tiled(CUtensorMap* map, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides,
                         const cuuint32_t* box, CUtensorMapSwizzle swizzle, CUtensorMapL2promotion l2)
{
    typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const EncodeFn encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        const bool ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) == cudaSuccess &&
                        q == cudaDriverEntryPointSuccess;
        if (!ok) cudaGetLastError();
        return ok ? reinterpret_cast<EncodeFn>(fn) : nullptr;
    }();
    if (!encode) return false;
    const cuuint32_t estr[3] = {1, 1, 1};
    auto go = [&] {
        return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), dims, strides, box, estr,
                      CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, l2, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    CUresult r = go();
    if (r == CUDA_ERROR_INVALID_CONTEXT) {
        // A driver call, which does not make a context current by itself as a launch does: a thread that has launched,
        // allocated and copied nothing yet has none.
        int device;
        if (cudaGetDevice(&device) != cudaSuccess || cudaSetDevice(device) != cudaSuccess) {
            cudaGetLastError();
            return false;
        }
        r = go();
    }
    return r == CUDA_SUCCESS;
}

// `rows` rows of `width` elements at `base`, boxes of box_rows x box_width.
inline bool encode_rows(CUtensorMap* map, const void* base, int width, int64_t rows, int box_width, int box_rows,
                        CUtensorMapSwizzle swizzle, CUtensorMapL2promotion l2)
{
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)width * 2};
    const cuuint32_t box[2] = {(cuuint32_t)box_width, (cuuint32_t)box_rows};
    return encode_tiled(map, base, 2, dims, strides, box, swizzle, l2);
}

// The same for each of `groups` groups, back to back: a box stays in its group and reads zeros behind the last row.
inline bool encode_groups(CUtensorMap* map, const void* base, int width, int64_t rows, int64_t groups, int box_width, int box_rows,
                          CUtensorMapSwizzle swizzle, CUtensorMapL2promotion l2)
{
    const cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)rows, (cuuint64_t)groups},
                     strides[2] = {(cuuint64_t)width * 2, (cuuint64_t)width * 2 * (cuuint64_t)rows};
    const cuuint32_t box[3] = {(cuuint32_t)box_width, (cuuint32_t)box_rows, 1};
    return encode_tiled(map, base, 3, dims, strides, box, swizzle, l2);
}

}  // namespace ckv
