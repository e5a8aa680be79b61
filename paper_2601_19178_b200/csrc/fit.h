// Internal declarations of the training side: sorted indices, router losses, gated pool lookup, and their gradients.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "ckv_internal.h"

namespace ckv {

#ifdef __CUDACC__
// A plain load.  (Kernels that are launched early wait for the ones before them, grid_dependency_wait; loads that promise that their
// memory does not change during the kernel, __ldg and those of const __restrict__ pointers, need not stay behind that wait.)
template <typename T>
__device__ __forceinline__ T ld(const T* p)
{
    return *p;
}
#endif

// Kernels of these calls that have been allowed how much shared memory on the current device, as far as this thread knows.
SmemGrants* fit_grants();
// launch_kernel with that record.  (A permission is lost with a device that the process resets: then the record starts anew.)
template <typename... P, typename... A>
cudaError_t launch_granted(cudaStream_t s, void (*fn)(P...), dim3 grid, int threads, size_t smem, A&&... args)
{
    SmemGrants* const g = fit_grants();
    const int known = g ? g->n : 0;
    cudaError_t e = launch_kernel(Launch{s, nullptr, g, true}, fn, grid, threads, smem, 1, args...);
    if (e == cudaErrorInvalidValue && known) {
        cudaGetLastError();
        g->n = 0;
        e = launch_kernel(Launch{s, nullptr, g, true}, fn, grid, threads, smem, 1, args...);
    }
    return e;
}

// Pieces of a caller's workspace, each on a 256-byte boundary.  A null base only adds up the size.
struct Carve {
    char* base;
    int64_t used = 0;
    explicit Carve(void* p) : base((char*)p) {}
    template <typename T>
    T* take(int64_t n)
    {
        T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used += (n * (int64_t)sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

// ---- kernels_sort.cu
int64_t sort_workspace(int64_t n, int G, int64_t m);
cudaError_t launch_sort_indices(int64_t n, int G, int64_t m, const int32_t* idx, int32_t* order, int32_t* offset, void* ws,
                                cudaStream_t s);

// ---- kernels_gather.cu
// out[i][g] = (user[i][g] | gate * pool[g][idx[i][g]]), gate = sigmoid(score[i][g]) or 1, rows of D elements, D - ds of them the user's
int64_t gather_workspace(int dtype, int64_t n, int G, int D, int ds, int64_t m);
cudaError_t launch_gather(int dtype, int64_t n, int G, int D, int ds, int64_t m, const void* pool, const int32_t* idx,
                          const void* user, const float* score, void* out, void* ws, cudaStream_t s);

// Sums of rows over the runs of equal entries in a sorted order, and what falls off on the way.
struct SegmentArgs {
    const int32_t* order;    // [G][n]
    const int32_t* offset;   // [G][m + 1]
    const void* rows;        // row of position i and group g at rows + i * stride + g * group_stride (elements)
    int64_t stride, group_stride;
    int64_t n, m;
    int G, width, skip;      // elements of a row, of which the first `skip` are not summed
    const float* score;      // [n][G] or null.  Weight of a row: sigmoid(score) if pool is given, else score itself; null: 1
    const void* pool;        // [G][m][width - skip]: d_score wanted; else null
    void* d_user;            // [n][G][skip] or null
    float* d_score;          // [n][G] or null
    float* sum;              // [G][m][width - skip]
    float* weight_sum;       // [G][m] or null: the sum of the weights
};
int64_t segment_workspace(int64_t n, int G, int width);
cudaError_t launch_segment_sum(int dtype, const SegmentArgs& a, void* ws, cudaStream_t s);

// ---- kernels_route_sweep.cu: passes over the score matrix
enum SweepMode { SWEEP_LSE, SWEEP_MEAN, SWEEP_R, SWEEP_DX, SWEEP_DW };
constexpr int kSweepPad = 384;      // rows of the arrays by position and by entry are rounded up to this
constexpr int kSweepMaxSplits = 64;
inline int64_t sweep_padded(int64_t n) { return (n + kSweepPad - 1) / kSweepPad * kSweepPad; }
struct SweepArgs {
    int64_t n, m, np, mp;           // positions, entries; both padded
    int G, splits, splits_dw;       // splits_dw: DW's, next to DX's
    bool join_here;                 // the last of a standing block's blocks joins their results
    const uint16_t *x, *W;          // [n][d], [G][m][d]
    const float *b, *h;             // [G][mp] bias (-inf behind the last entry); h
    float *nl, *nr;                 // [G][np] -lse (-inf: no weight), which LSE leaves; -r, which R leaves
    const uint16_t* b_step;         // b and nl as operands of a product, see put_step
    uint16_t* nl_step;
    float* part;    // LSE: float2 (maximum, sum) [splits][G][np]; MEAN [splits][G][mp]; R [splits][G][np]; DX [splits][n][d]
    float *part_dw, *part2;  // DW [splits_dw][G][m][d], and the sums of T [splits_dw][G][mp]
    unsigned* ticket;   // LSE, MEAN, R: zero; blocks that are done, of each standing block (and group); MEAN: and of each group
    // LSE, MEAN: indices, scores, results; per block of kSweepPad positions and group the positions that take part, those of them that have
    // a weight (scores that are not all -inf) and the sum of -log sigmoid(score); per block of as many entries the balance loss's part
    const int32_t* idx;
    const float *score, *spoilt;  // spoilt [n]: NaN where lse is to be that, else 0
    float *lse, *mean, *loss;
    int32_t *rows_part, *live_part;
    double *peak_part, *balance_part;
    // what is joined to DX and DW: the picked entry's coefficient [n][G], and the sums over an entry's positions of what it multiplies and of itself
    const float *ds, *sum, *wsum;
};
inline int64_t sweep_blocks(int64_t rows) { return sweep_padded(rows) / kSweepPad; }
// tickets of a pass
int64_t sweep_tickets(int64_t n, int G, int d, int64_t m, int mode);
#ifdef __CUDACC__
// A number as three bf16 parts whose sum it is.
__device__ __forceinline__ uint2 bf16_parts(float v)
{
    const uint32_t hi = (__float_as_uint(v) & 0xffff0000u) | (v != v ? 0x400000u : 0u);  // (a NaN whose upper half alone would be an infinity)
    const float r1 = isfinite(v) ? v - __uint_as_float(hi) : 0.f;
    const uint32_t mid = __float_as_uint(r1) & 0xffff0000u, lo = __float_as_uint(r1 - __uint_as_float(mid));
    return make_uint2((hi >> 16) | mid, lo >> 16);
}
// Those parts as a row of a K-major operand without swizzle (16 elements per row: 8 rows of 16 bytes, of which the first six hold the parts,
// then the rows' zero halves).
__device__ __forceinline__ void put_step(uint16_t* step, int64_t row, float v)
{
    const uint2 parts = bf16_parts(v);
    uint4* const to = reinterpret_cast<uint4*>(step) + (row >> 3) * 16 + (row & 7);
    to[0] = make_uint4(parts.x, parts.y, 0, 0);
    to[8] = make_uint4(0, 0, 0, 0);
}
#endif
int sweep_splits(int64_t n, int G, int d, int64_t m, int mode);
cudaError_t launch_sweep(int mode, int d, SweepArgs& a, cudaStream_t s);  // LSE, MEAN, R with a.splits, and what joins their partial results
cudaError_t launch_sweep_grad(int d, SweepArgs& a, cudaStream_t s);       // DX with a.splits, DW with a.splits_dw

// ---- kernels_route_loss.cu
struct RouteLossArgs {
    int64_t n, m;
    int G, d;
    const void *x, *W;
    const float* bias;
    const int32_t* idx;
    float *loss, *lse, *score, *mean;  // outputs of the forward pass, inputs of the gradient
};
int64_t route_loss_workspace(int64_t n, int G, int d, int64_t m);
// kNoRoom (an error that no launch reports) where the workspace is smaller than that
constexpr cudaError_t kNoRoom = cudaErrorInvalidPitchValue;
cudaError_t launch_route_loss(const RouteLossArgs& a, void* ws, int64_t bytes, cudaStream_t s);
struct RouteGradArgs {
    const int32_t *order, *offset;
    float w_balance, w_peak;
    const float* d_score;  // or null
    void *dx, *dW;
    float* dbias;          // or null
};
int64_t route_grad_workspace(int64_t n, int G, int d, int64_t m);
cudaError_t launch_route_grad(const RouteLossArgs& a, const RouteGradArgs& b, void* ws, int64_t bytes, cudaStream_t s);

}  // namespace ckv
