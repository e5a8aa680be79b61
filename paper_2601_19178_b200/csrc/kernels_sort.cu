// Positions ordered by the pool entry they picked: a stable counting sort per group.
//
//   order[g]  = positions i by (key(i), i), key = idx[i][g] if it lies in [0, m), else m (no entry: behind all others)
//   offset[g][j] = number of positions of the group with a key below j, j = 0..m
//
// The positions are cut into chunks.  A chunk counts its keys in shared memory (one word per key: `table[g][chunk][key]`),
// the counts are added up over the chunks of a group and over the keys, and every chunk then places its positions in their order,
// so that equal keys keep it and the result does not depend on how blocks are scheduled.  Keys of more than kDigitBits
// bits are sorted digit by digit, the low ones first.
#include <algorithm>

#include "fit.h"
#include "ptx_helpers.cuh"

namespace ckv {
namespace {

constexpr int kDigitBits = 15;

// A pass over the keys: from the indices (first pass) or from the pass before.
struct Pass {
    const int32_t* idx;    // [n][G], or null
    const uint32_t* key;   // [G][n] keys and the positions they belong to, of the pass before
    const int32_t* val;
    uint32_t* key_out;     // [G][n], or null: nothing reads them any more
    int32_t* val_out;
    int64_t n, m, chunk;
    int G, chunks, bins, shift;
};
__device__ __forceinline__ uint32_t key_at(const Pass& p, int g, int64_t i)
{
    if (!p.idx) return __ldg(p.key + (int64_t)g * p.n + i);
    const int32_t v = __ldg(p.idx + i * p.G + g);
    return v >= 0 && v < p.m ? (uint32_t)v : (uint32_t)p.m;
}
__device__ __forceinline__ int digit_of(const Pass& p, uint32_t key) { return (int)((key >> p.shift) & (uint32_t)((1 << kDigitBits) - 1)); }

__global__ void __launch_bounds__(256) count_kernel(const Pass p, int32_t* __restrict__ table)
{
    extern __shared__ int32_t bins[];
    const int g = blockIdx.y;
    for (int j = threadIdx.x; j < p.bins; j += 256) bins[j] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * p.chunk, end = min(begin + p.chunk, p.n);
    for (int64_t i = begin + threadIdx.x; i < end; i += 256) atomicAdd(bins + digit_of(p, key_at(p, g, i)), 1);
    __syncthreads();
    int32_t* t = table + ((int64_t)g * p.chunks + blockIdx.x) * p.bins;
    for (int j = threadIdx.x; j < p.bins; j += 256) t[j] = bins[j];
}

// table[g][c][j] becomes the count of the chunks before c, total[g][j] that of all
__global__ void __launch_bounds__(256) chunk_scan_kernel(int32_t* __restrict__ table, int32_t* __restrict__ total, int chunks, int bins)
{
    const int j = blockIdx.x * 256 + threadIdx.x, g = blockIdx.y;
    if (j >= bins) return;
    int32_t* t = table + (int64_t)g * chunks * bins + j;
    int32_t sum = 0;
    for (int c = 0; c < chunks; ++c, t += bins) {
        const int32_t v = *t;
        *t = sum;
        sum += v;
    }
    total[(int64_t)g * bins + j] = sum;
}

// exclusive prefix sums of a group's totals, in place; copied to offset (whose rows have as many entries) if given
__global__ void __launch_bounds__(1024) bin_scan_kernel(int32_t* __restrict__ total, int32_t* __restrict__ offset, int bins)
{
    __shared__ int32_t warp_sum[32];
    const int g = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int32_t* t = total + (int64_t)g * bins;
    int32_t carry = 0;
    for (int j0 = 0; j0 < bins; j0 += 1024) {
        const int j = j0 + threadIdx.x;
        const int32_t v = j < bins ? t[j] : 0;
        int32_t s = v;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int32_t o = __shfl_up_sync(0xffffffffu, s, d);
            if (lane >= d) s += o;
        }
        if (lane == 31) warp_sum[warp] = s;
        __syncthreads();
        int32_t before = 0, all = 0;
        for (int w = 0; w < 32; ++w) {
            if (w < warp) before += warp_sum[w];
            all += warp_sum[w];
        }
        __syncthreads();
        if (j < bins) {
            t[j] = carry + before + s - v;
            if (offset) offset[(int64_t)g * bins + j] = t[j];
        }
        carry += all;
    }
}

// One warp per chunk: 32 positions at a time, the lanes with equal keys in the order of their positions.
__global__ void __launch_bounds__(32) place_kernel(const Pass p, const int32_t* __restrict__ table, const int32_t* __restrict__ base)
{
    extern __shared__ int32_t next[];
    const int g = blockIdx.y, lane = threadIdx.x;
    const int32_t *t = table + ((int64_t)g * p.chunks + blockIdx.x) * p.bins, *b = base + (int64_t)g * p.bins;
    for (int j = lane; j < p.bins; j += 32) next[j] = t[j] + b[j];
    __syncwarp();
    const int64_t begin = blockIdx.x * p.chunk, end = min(begin + p.chunk, p.n);
    for (int64_t i0 = begin; i0 < end; i0 += 32) {
        const int64_t i = i0 + lane;
        const bool real = i < end;
        const uint32_t key = real ? key_at(p, g, i) : 0;
        const int d = real ? digit_of(p, key) : -1;
        const unsigned same = __match_any_sync(0xffffffffu, d);
        const int leader = __ffs(same) - 1;
        int32_t at = 0;
        if (real && lane == leader) at = atomicAdd(next + d, __popc(same));
        at = __shfl_sync(0xffffffffu, at, leader) + __popc(same & ((1u << lane) - 1));
        if (real) {
            const int64_t o = (int64_t)g * p.n + at;
            p.val_out[o] = p.val ? p.val[(int64_t)g * p.n + i] : (int32_t)i;
            if (p.key_out) p.key_out[o] = key;
        }
    }
}

// offset[g][j] = number of sorted keys below j
__global__ void __launch_bounds__(256) bounds_kernel(const uint32_t* __restrict__ key, int32_t* __restrict__ offset, int64_t n, int64_t m)
{
    const int64_t j = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (j > m) return;
    const uint32_t* k = key + (int64_t)blockIdx.y * n;
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if ((int64_t)k[mid] < j) lo = mid + 1;
        else hi = mid;
    }
    offset[(int64_t)blockIdx.y * (m + 1) + j] = (int32_t)lo;
}

int bits_of(int64_t m)  // of the largest key, m
{
    int b = 1;
    while (m >> b) ++b;
    return b;
}
int passes_of(int64_t m) { return (bits_of(m) + kDigitBits - 1) / kDigitBits; }
int bins_of(int64_t m) { return passes_of(m) == 1 ? (int)m + 1 : 1 << kDigitBits; }
int64_t chunk_of(int64_t n, int G, int64_t m)
{
    int64_t c = 1024;
    while (c * 592 < n * G || 2 * c < bins_of(m)) c *= 2;
    return c;
}

struct SortSpace {
    int32_t *table, *total, *val[2];
    uint32_t* key[2];
    int64_t bytes;
    SortSpace(void* ws, int64_t n, int G, int64_t m)
    {
        Carve c(ws);
        const int64_t chunks = (n + chunk_of(n, G, m) - 1) / chunk_of(n, G, m);
        table = c.take<int32_t>(chunks * G * bins_of(m));
        total = c.take<int32_t>((int64_t)G * bins_of(m));
        val[0] = val[1] = nullptr;
        key[0] = key[1] = nullptr;
        if (passes_of(m) > 1)
            for (int i = 0; i < 2; ++i) {
                key[i] = c.take<uint32_t>(n * G);
                val[i] = c.take<int32_t>(n * G);
            }
        bytes = c.used;
    }
};

}  // namespace

int64_t sort_workspace(int64_t n, int G, int64_t m) { return SortSpace(nullptr, n, G, m).bytes; }

cudaError_t launch_sort_indices(int64_t n, int G, int64_t m, const int32_t* idx, int32_t* order, int32_t* offset, void* ws,
                                cudaStream_t s)
{
    const SortSpace sp(ws, n, G, m);
    const int passes = passes_of(m), bins = bins_of(m);
    const Launch l{s, nullptr, nullptr};
    Pass p{};
    p.n = n;
    p.m = m;
    p.G = G;
    p.chunk = chunk_of(n, G, m);
    p.chunks = (int)((n + p.chunk - 1) / p.chunk);
    p.bins = bins;
    for (int i = 0; i < passes; ++i) {
        p.shift = i * kDigitBits;
        p.idx = i == 0 ? idx : nullptr;
        p.key = i == 0 ? nullptr : sp.key[(i - 1) & 1];
        p.val = i == 0 ? nullptr : sp.val[(i - 1) & 1];
        p.key_out = passes == 1 ? nullptr : sp.key[i & 1];
        p.val_out = i + 1 == passes ? order : sp.val[i & 1];
        const dim3 grid((unsigned)p.chunks, (unsigned)G);
        cudaError_t e = p.chunks ? launch_kernel(l, count_kernel, grid, 256, bins * 4, 1, p, sp.table) : cudaSuccess;
        if (e == cudaSuccess)
            e = launch_kernel(l, chunk_scan_kernel, dim3((bins + 255) / 256, (unsigned)G), 256, 0, 1, sp.table, sp.total, p.chunks, bins);
        if (e == cudaSuccess)
            e = launch_kernel(l, bin_scan_kernel, dim3((unsigned)G), 1024, 0, 1, sp.total, passes == 1 ? offset : nullptr, bins);
        if (e == cudaSuccess && p.chunks) e = launch_kernel(l, place_kernel, grid, 32, bins * 4, 1, p, sp.table, sp.total);
        if (e != cudaSuccess) return e;
    }
    if (passes > 1)
        return launch_kernel(l, bounds_kernel, dim3((unsigned)((m + 256) / 256), (unsigned)G), 256, 0, 1, sp.key[(passes - 1) & 1],
                             offset, n, m);
    return cudaSuccess;
}

}  // namespace ckv
