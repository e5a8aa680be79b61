// Gated lookup of pool rows (Eq. Kc, training branch) and its gradient.
//
//   out[i][g]   = (user[i][g] | s_i pool[g][I_i]),  s = sigmoid(score) or 1; a position without an entry gets zeros
//   d_pool[g][j] = sum over the positions of entry j, in their order, of s_i d_out[i][g][skip:]
//   d_user = d_out[:skip],  d_score_i = s_i (1 - s_i) <pool[g][I_i], d_out[i][g][skip:]>
#include <cuda_bf16.h>

#include <algorithm>

#include "fit.h"
#include "ptx_helpers.cuh"

namespace ckv {
namespace {

template <typename E>
__device__ __forceinline__ float widen(E v);
template <>
__device__ __forceinline__ float widen<float>(float v) { return v; }
template <>
__device__ __forceinline__ float widen<uint16_t>(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
template <typename E>
__device__ __forceinline__ E narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ uint16_t narrow<uint16_t>(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

template <typename E>
__global__ void __launch_bounds__(256) gather_kernel(int64_t rows, int G, int D, int skip, int64_t m, const E* __restrict__ pool,
                                                     const int32_t* __restrict__ idx, const E* __restrict__ user,
                                                     const float* __restrict__ score, E* __restrict__ out)
{
    const int ds = D - skip;
    for (int64_t e = blockIdx.x * (int64_t)256 + threadIdx.x; e < rows * D; e += (int64_t)gridDim.x * 256) {
        const int64_t r = e / D;
        const int c = (int)(e - r * D), g = (int)(r % G);
        if (c < skip) {
            out[e] = user[r * skip + c];
            continue;
        }
        const int32_t j = idx[r];
        float v = 0.f;
        if (j >= 0 && j < m) {
            v = widen(pool[((int64_t)g * m + j) * ds + (c - skip)]);
            if (score) v *= sigmoid(score[r]);
        }
        out[e] = narrow<E>(v);
    }
}

// ---- sums over runs of equal entries ---------------------------------------------------------------------------
// One warp per chunk of the sorted positions of a group, whatever the entries: runs that lie inside the chunk are written,
// the one that began before it and the one that goes on behind it leave a partial sum (head, tail), which join_kernel adds up
// in the order of the chunks.  Nothing depends on the order in which warps run.
constexpr int kChunk = 64, kWarps = 4, kMaxCols = 4;  // widths up to 32 kMaxCols

template <typename E>
__global__ void __launch_bounds__(32 * kWarps) segment_kernel(const SegmentArgs a, float* __restrict__ part, float* __restrict__ wpart, int chunks)
{
    const int lane = threadIdx.x & 31, g = blockIdx.y;
    const int c = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (c >= chunks) return;
    const int ds = a.width - a.skip;
    const int32_t *order = a.order + (int64_t)g * a.n, *offset = a.offset + (int64_t)g * (a.m + 1);
    const int64_t begin = (int64_t)c * kChunk, end = min(begin + kChunk, a.n);
    // the entry of the first position: the last j with offset[j] <= begin (m: no entry)
    int64_t lo = 0, hi = a.m;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) / 2;
        if (offset[mid] <= begin) lo = mid;
        else hi = mid - 1;
    }
    int64_t j = lo, run_end = j < a.m ? offset[j + 1] : a.n;
    bool head = offset[j] < begin;
    float acc[kMaxCols] = {}, row_pool[kMaxCols] = {}, wsum = 0.f;
    float* const p = part + ((int64_t)g * chunks + c) * 2 * a.width;
    float* const wp = wpart + ((int64_t)g * chunks + c) * 2;
    auto fetch_pool = [&] {
#pragma unroll
        for (int q = 0; q < kMaxCols; ++q) {
            const int col = lane + 32 * q;
            row_pool[q] = a.pool && j < a.m && col >= a.skip && col < a.width
                              ? widen(((const E*)a.pool)[((int64_t)g * a.m + j) * ds + col - a.skip]) : 0.f;
        }
    };
    auto flush = [&](bool tail) {
        if (j < a.m) {
#pragma unroll
            for (int q = 0; q < kMaxCols; ++q) {
                const int col = lane + 32 * q;
                if (col < a.skip || col >= a.width) continue;
                if (head) p[col] = acc[q];
                else if (tail) p[a.width + col] = acc[q];
                else a.sum[((int64_t)g * a.m + j) * ds + col - a.skip] = acc[q];
            }
            if (a.weight_sum && lane == 0) {
                if (head) wp[0] = wsum;
                else if (tail) wp[1] = wsum;
                else a.weight_sum[(int64_t)g * a.m + j] = wsum;
            }
        }
#pragma unroll
        for (int q = 0; q < kMaxCols; ++q) acc[q] = 0.f;
        wsum = 0.f;
        head = false;
    };
    fetch_pool();
    for (int64_t t = begin; t < end; ++t) {
        if (t >= run_end) {
            flush(false);
            do {
                ++j;
                run_end = j < a.m ? offset[j + 1] : a.n;
            } while (t >= run_end);
            fetch_pool();
        }
        const int64_t i = order[t];
        if (i < 0 || i >= a.n) continue;  // not an order
        const E* row = (const E*)a.rows + i * a.stride + g * a.group_stride;
        const float sc = a.score ? a.score[i * a.G + g] : 0.f;
        const float w = !a.score ? 1.f : a.pool ? sigmoid(sc) : sc;
        float dot = 0.f;
#pragma unroll
        for (int q = 0; q < kMaxCols; ++q) {
            const int col = lane + 32 * q;
            if (col >= a.width) continue;
            const E raw = row[col];
            const float v = widen(raw);
            if (col < a.skip) {
                if (a.d_user) ((E*)a.d_user)[(i * a.G + g) * a.skip + col] = raw;
            } else {
                acc[q] = fmaf(w, v, acc[q]);
                dot = fmaf(row_pool[q], v, dot);
            }
        }
        wsum += w;
        if (a.d_score) {
#pragma unroll
            for (int d = 16; d > 0; d /= 2) dot += __shfl_xor_sync(0xffffffffu, dot, d);
            if (lane == 0) a.d_score[i * a.G + g] = j < a.m ? dot * w * sigmoid(-sc) : 0.f;
        }
    }
    flush(run_end > end);
}

// Blocks of the first kind: the run that goes on behind chunk c and began in it.  Of the second: entries without a position.
__global__ void __launch_bounds__(128) join_kernel(const SegmentArgs a, const float* __restrict__ part, const float* __restrict__ wpart, int chunks)
{
    const int g = blockIdx.y, ds = a.width - a.skip, col = a.skip + (int)threadIdx.x;
    const int32_t* offset = a.offset + (int64_t)g * (a.m + 1);
    if ((int)blockIdx.x < chunks - 1) {
        const int c = blockIdx.x;
        const int64_t end = (int64_t)(c + 1) * kChunk;
        int64_t lo = 0, hi = a.m;
        while (lo < hi) {
            const int64_t mid = (lo + hi + 1) / 2;
            if (offset[mid] < end) lo = mid;
            else hi = mid - 1;
        }
        if (lo >= a.m || offset[lo + 1] <= end || offset[lo] < end - kChunk) return;
        const int last = min((offset[lo + 1] - 1) / kChunk, chunks - 1);
        if (col < a.width) {
            float sum = part[(((int64_t)g * chunks + c) * 2 + 1) * a.width + col];
            for (int k = c + 1; k <= last; ++k) sum += part[((int64_t)g * chunks + k) * 2 * a.width + col];
            a.sum[((int64_t)g * a.m + lo) * ds + threadIdx.x] = sum;
        }
        if (a.weight_sum && threadIdx.x == 0) {
            float sum = wpart[((int64_t)g * chunks + c) * 2 + 1];
            for (int k = c + 1; k <= last; ++k) sum += wpart[((int64_t)g * chunks + k) * 2];
            a.weight_sum[(int64_t)g * a.m + lo] = sum;
        }
        return;
    }
    const int64_t first = (int64_t)((int)blockIdx.x - max(chunks - 1, 0)) * 32;
    for (int64_t j = first; j < min(first + 32, a.m); ++j) {
        if (offset[j] != offset[j + 1]) continue;
        if (col < a.width) a.sum[((int64_t)g * a.m + j) * ds + threadIdx.x] = 0.f;
        if (a.weight_sum && threadIdx.x == 0) a.weight_sum[(int64_t)g * a.m + j] = 0.f;
    }
}

struct SegmentSpace {
    float *part, *wpart;
    int64_t bytes;
    SegmentSpace(void* ws, int64_t n, int G, int width)
    {
        Carve c(ws);
        const int64_t chunks = (n + kChunk - 1) / kChunk;
        part = c.take<float>(chunks * G * 2 * width);
        wpart = c.take<float>(chunks * G * 2);
        bytes = c.used;
    }
};

}  // namespace

cudaError_t launch_gather(int dtype, int64_t n, int G, int D, int ds, int64_t m, const void* pool, const int32_t* idx,
                          const void* user, const float* score, void* out, cudaStream_t s)
{
    const int64_t blocks = std::min<int64_t>((n * G * D + 255) / 256, 148 * 32);
    const Launch l{s, nullptr, nullptr};
    if (dtype == CKV_F32)
        return launch_kernel(l, gather_kernel<float>, dim3((unsigned)blocks), 256, 0, 1, n * G, G, D, D - ds, m, (const float*)pool, idx,
                             (const float*)user, score, (float*)out);
    return launch_kernel(l, gather_kernel<uint16_t>, dim3((unsigned)blocks), 256, 0, 1, n * G, G, D, D - ds, m, (const uint16_t*)pool,
                         idx, (const uint16_t*)user, score, (uint16_t*)out);
}

int64_t segment_workspace(int64_t n, int G, int width) { return SegmentSpace(nullptr, n, G, width).bytes; }

cudaError_t launch_segment_sum(int dtype, const SegmentArgs& a, void* ws, cudaStream_t s)
{
    const SegmentSpace sp(ws, a.n, a.G, a.width);
    const int chunks = (int)((a.n + kChunk - 1) / kChunk);
    const Launch l{s, nullptr, nullptr};
    cudaError_t e = cudaSuccess;
    if (chunks > 0)
        e = launch_kernel(l, dtype == CKV_F32 ? segment_kernel<float> : segment_kernel<uint16_t>,
                          dim3((unsigned)((chunks + kWarps - 1) / kWarps), (unsigned)a.G), 32 * kWarps, 0, 1, a, sp.part, sp.wpart, chunks);
    if (e == cudaSuccess)
        e = launch_kernel(l, join_kernel, dim3((unsigned)(std::max(chunks - 1, 0) + (a.m + 31) / 32), (unsigned)a.G), 128, 0, 1, a, sp.part,
                          sp.wpart, chunks);
    return e;
}

}  // namespace ckv
