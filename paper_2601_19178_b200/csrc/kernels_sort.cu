// Positions ordered by the pool entry they picked: a stable counting sort per group.
//
//   order[g]  = positions i by (key(i), i), key = idx[i][g] if it lies in [0, m), else m (no entry: behind all others)
//   offset[g][j] = number of positions of the group with a key below j, j = 0..m
//
// Up to kBlockSort positions a block sorts a group in shared memory.  More are cut into chunks: a chunk counts its keys in shared memory (one
// word per key: `table[g][chunk][key]`), the counts are added up over the chunks of a group and over the keys, and a warp
// per chunk then places its positions in their order, so that equal keys keep it and the result does not depend on how
// blocks are scheduled.  Keys of more than kDigitBits bits are sorted digit by digit, the low ones first.
#include <algorithm>
#include <cmath>

#include "fit.h"
#include "ptx_helpers.cuh"

namespace ckv {
namespace {

constexpr int kDigitBits = 14, kOnePassBins = 25000, kBlockSort = 8192, kBlockThreads = 512;
constexpr int kAhead = 8;  // batches of 32 positions whose keys a placing warp has on their way

__device__ __forceinline__ uint32_t key_of(int32_t v, int64_t m) { return v >= 0 && v < m ? (uint32_t)v : (uint32_t)m; }

// A pass over the keys: from the indices (first pass) or from the pass before.
struct Pass {
    const int32_t* idx;    // [n][G], or null
    uint32_t* key;         // [G][n] keys (the first pass writes them) and the positions they belong to (null: 0, 1, ...)
    const int32_t* val;
    uint32_t* key_out;     // [G][n], or null: nothing reads them any more
    int32_t* val_out;
    int64_t n, m, chunk;
    int G, chunks, bins, stride, shift, mask;  // stride: of a row of the table, a multiple of four; mask: of a digit
};
__device__ __forceinline__ int digit_of(uint32_t key, const Pass& p) { return (int)(key >> p.shift) & p.mask & 0x7fff; }

// Bound by shared-memory atomics (the data pipe 65 % busy) and the strided indices: 1048576 x 8 positions, 4096 entries 24 us.
__global__ void __launch_bounds__(256) count_kernel(const Pass p, int32_t* table)
{
    extern __shared__ int32_t bins[];
    const int g = blockIdx.y;
    for (int j = threadIdx.x; j < p.stride; j += 256) bins[j] = 0;
    grid_dependency_wait();
    __syncthreads();
    const int64_t begin = blockIdx.x * p.chunk, end = min(begin + p.chunk, p.n);
    uint32_t* keys = p.key + (int64_t)g * p.n;
#pragma unroll 8
    for (int64_t i = begin + threadIdx.x; i < end; i += 256) {
        uint32_t k;
        if (p.idx) keys[i] = k = key_of(ld(p.idx + i * p.G + g), p.m);
        else k = keys[i];
        atomicAdd(bins + digit_of(k, p), 1);
    }
    __syncthreads();
    int32_t* t = table + ((int64_t)g * p.chunks + blockIdx.x) * p.stride;
    for (int j = threadIdx.x; j < p.stride; j += 256) t[j] = bins[j];
}

// table[g][c][j] becomes the count of the chunks before c, total[g][j] that of all
constexpr int kScanAhead = 16;
__global__ void __launch_bounds__(128) chunk_scan_kernel(int32_t* table, int32_t* total, int chunks, int stride)
{
    const int j = blockIdx.x * 128 + threadIdx.x, g = blockIdx.y;
    grid_dependency_wait();
    if (j >= stride) return;
    int32_t* t = table + (int64_t)g * chunks * stride + j;
    int32_t sum = 0;
    for (int c0 = 0; c0 < chunks; c0 += kScanAhead) {
        int32_t v[kScanAhead];
#pragma unroll
        for (int k = 0; k < kScanAhead; ++k) v[k] = c0 + k < chunks ? t[(int64_t)(c0 + k) * stride] : 0;
#pragma unroll
        for (int k = 0; k < kScanAhead; ++k) {
            if (c0 + k < chunks) t[(int64_t)(c0 + k) * stride] = sum;
            sum += v[k];
        }
    }
    total[(int64_t)g * stride + j] = sum;
}

// Exclusive prefix sum over a block's threads of one number each; *all: the sum of all.
template <int THREADS>
__device__ __forceinline__ int32_t block_prefix(int32_t v, int32_t* all)
{
    __shared__ int32_t warp_sum[THREADS / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int32_t s = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int32_t o = __shfl_up_sync(0xffffffffu, s, d);
        if (lane >= d) s += o;
    }
    __syncthreads();
    if (lane == 31) warp_sum[warp] = s;
    __syncthreads();
    int32_t w = lane < THREADS / 32 ? warp_sum[lane] : 0;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int32_t o = __shfl_up_sync(0xffffffffu, w, d);
        if (lane >= d) w += o;
    }
    *all = __shfl_sync(0xffffffffu, w, 31);
    const int32_t before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    return s - v + (warp ? before : 0);
}

// exclusive prefix sums of a group's totals, in place; copied to offset (rows of `bins`) if given
__global__ void __launch_bounds__(1024) bin_scan_kernel(int32_t* total, int32_t* offset, int bins, int stride)
{
    const int g = blockIdx.x;
    int32_t* t = total + (int64_t)g * stride;
    int32_t carry = 0;
    grid_dependency_wait();
    for (int j0 = 0; j0 < bins; j0 += 4096) {
        const int j = j0 + threadIdx.x * 4;
        const int4 v = j < stride ? *reinterpret_cast<int4*>(t + j) : make_int4(0, 0, 0, 0);
        int32_t all;
        int32_t at = carry + block_prefix<1024>(v.x + v.y + v.z + v.w, &all);
        const int32_t o[4] = {at, at + v.x, at + v.x + v.y, at + v.x + v.y + v.z};
        if (j < stride) *reinterpret_cast<int4*>(t + j) = make_int4(o[0], o[1], o[2], o[3]);
        if (offset)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (j + q < bins) offset[(int64_t)g * bins + j + q] = o[q];
        carry += all;
    }
}

// One warp's turn with 32 positions: the place of each, next[] moved on.  Lanes with equal keys (`same`) stay in order.  The warp has
// next[] to itself: a read, and a write by one lane of each key.
__device__ __forceinline__ int32_t take_places(volatile int32_t* next, int d, unsigned same)  // d < 0: none
{
    const int lane = threadIdx.x & 31;
    int32_t at = 0;
    if (d >= 0) at = next[d];
    __syncwarp();  // (every lane has read before one writes)
    if (d >= 0 && lane == __ffs(same) - 1) next[d] = at + __popc(same);
    __syncwarp();
    return at + __popc(same & ((1u << lane) - 1));
}

// A chunk's positions to their places, by one warp (the block's others help to fetch next[]).  Bound by its turns, of which a match
// instruction is the longest part (its time grows with the number of different keys in the warp; 0.3 us a turn): 1048576 x 8
// positions, 4096 entries 68 us of 109.  (Lanes that find each other through a word per key, as in block_sort_kernel, halve a turn, but with
// half as many warps to an SM: 85; two to eight warps with a part of a larger chunk each, whose parts the block counts first, no
// less, for the match instructions of an SM take turns; votes on the 13 bits of a key instead of the match 113.)
__global__ void __launch_bounds__(128) place_kernel(const Pass p, const int32_t* table, const int32_t* base)
{
    extern __shared__ __align__(16) int32_t next[];
    const int g = blockIdx.y, lane = threadIdx.x & 31;
    grid_dependency_wait();
    const int32_t *t = table + ((int64_t)g * p.chunks + blockIdx.x) * p.stride, *b = base + (int64_t)g * p.stride;
#pragma unroll 4
    for (int j = threadIdx.x * 4; j < p.stride; j += 512) {
        const int4 x = ld(reinterpret_cast<const int4*>(t + j)), y = ld(reinterpret_cast<const int4*>(b + j));
        *reinterpret_cast<int4*>(next + j) = make_int4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
    }
    __syncthreads();
    if (threadIdx.x >= 32) return;
    const int64_t begin = blockIdx.x * p.chunk, end = min(begin + p.chunk, p.n), row = (int64_t)g * p.n;
    uint32_t key[kAhead];
    int32_t val[kAhead];
    auto fetch = [&](int64_t i0) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t i = i0 + 32 * k + lane;
            key[k] = i < end ? ld(p.key + row + i) : 0xffffffffu;
            val[k] = !p.val ? (int32_t)i : i < end ? ld(p.val + row + i) : 0;
        }
    };
    fetch(begin);
    for (int64_t i0 = begin; i0 < end; i0 += 32 * kAhead) {
        uint32_t k_now[kAhead];
        int32_t v_now[kAhead], at[kAhead], d[kAhead];
        unsigned same[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            k_now[k] = key[k];
            v_now[k] = val[k];
        }
        fetch(i0 + 32 * kAhead);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            d[k] = i0 + 32 * k + lane < end ? digit_of(k_now[k], p) : -1;
            same[k] = __match_any_sync(0xffffffffu, d[k]);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) at[k] = take_places(next, d[k], same[k]);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (d[k] < 0) continue;
            p.val_out[row + at[k]] = v_now[k];
            if (p.key_out) p.key_out[row + at[k]] = k_now[k];
        }
    }
}

// A key's word pair: the lanes that hold it in the turn at hand, and the place of its next position.
struct Slot {
    unsigned lanes;
    int32_t next;
};
// take_places for lanes that find each other through the slots.
__device__ __forceinline__ int32_t take_places(Slot* slots, int d)  // d < 0: none
{
    const int lane = threadIdx.x & 31;
    if (d >= 0) atomicOr(&slots[d].lanes, 1u << lane);
    __syncwarp();
    Slot s{0, 0};
    if (d >= 0) {
        const unsigned long long v = *reinterpret_cast<volatile unsigned long long*>(slots + d);
        s.lanes = (unsigned)v;
        s.next = (int32_t)(v >> 32);
    }
    __syncwarp();
    if (d >= 0 && lane == __ffs(s.lanes) - 1)
        *reinterpret_cast<volatile unsigned long long*>(slots + d) = (unsigned long long)(uint32_t)(s.next + __popc(s.lanes)) << 32;
    __syncwarp();
    return s.next + __popc(s.lanes & ((1u << lane) - 1));
}

// The whole sort of a group by one block, of which one warp places: 8000 positions x 8 groups x 300 entries 29 us (55 with a match).
__global__ void __launch_bounds__(kBlockThreads) block_sort_kernel(int n, int G, int64_t m, const int32_t* idx,
                                                                   int32_t* order, int32_t* offset)
{
    extern __shared__ __align__(16) Slot slots[];
    const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 31, bins = (int)m + 1;
    uint16_t* keys = reinterpret_cast<uint16_t*>(slots + ((bins + 3) & ~3));
    for (int j = tid; j < bins; j += kBlockThreads) slots[j] = Slot{0, 0};
    grid_dependency_wait();
    __syncthreads();
#pragma unroll 4
    for (int i = tid; i < n; i += kBlockThreads) {
        const int k = (int)key_of(ld(idx + (int64_t)i * G + g), m);
        keys[i] = (uint16_t)k;
        atomicAdd(&slots[k].next, 1);
    }
    __syncthreads();
    int32_t carry = 0;
    for (int j0 = 0; j0 < bins; j0 += kBlockThreads) {
        const int j = j0 + tid;
        int32_t all;
        const int32_t at = carry + block_prefix<kBlockThreads>(j < bins ? slots[j].next : 0, &all);
        if (j < bins) {
            slots[j].next = at;
            offset[(int64_t)g * bins + j] = at;
        }
        carry += all;
    }
    __syncthreads();
    if (tid >= 32) return;
#pragma unroll 4
    for (int i0 = 0; i0 < n; i0 += 32) {
        const int i = i0 + lane;
        const int d = i < n ? keys[i] : -1;
        const int32_t at = take_places(slots, d);
        if (i < n) order[(int64_t)g * n + at] = i;
    }
}

// offset[g][j] = number of sorted keys below j
__global__ void __launch_bounds__(256) bounds_kernel(const uint32_t* key, int32_t* offset, int64_t n, int64_t m)
{
    const int64_t j = blockIdx.x * (int64_t)256 + threadIdx.x;
    grid_dependency_wait();
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
int passes_of(int64_t m) { return m < kOnePassBins ? 1 : (bits_of(m) + kDigitBits - 1) / kDigitBits; }
int digit_bits(int64_t m) { return (bits_of(m) + passes_of(m) - 1) / passes_of(m); }
int bins_of(int64_t m) { return passes_of(m) == 1 ? (int)m + 1 : 1 << digit_bits(m); }
int stride_of(int64_t m) { return (bins_of(m) + 3) & ~3; }
bool by_block(int64_t n, int64_t m) { return n <= kBlockSort && passes_of(m) == 1; }
// Positions of a chunk, a power of two: the number with the shortest run, in microseconds.  A turn of 32 positions takes a warp 0.3, an SM holds as
// many chunks as their counts leave room for (at most 16), a chunk's counts are written, read, written and read, at some 1.5 TB/s,
// and adding up sixteen chunks of a group takes 1.  (1048576 x 8 positions, 4000 entries: 111 us with chunks of 8192, 133 with 4096, 168
// with 16384; 200000 x 2, 1000 entries: 24 with 1024, 27 with 2048; 50000 x 4, 5000 entries: 25 with 1024, 42 with 4096.)
int64_t chunk_of(int64_t n, int G, int64_t m)
{
    int64_t best = 512;
    double best_t = 1e300;
    for (int64_t c = 512; c <= 32768; c *= 2) {
        const double chunks = (double)((n + c - 1) / c) * G, room = 148.0 * std::min(16, 220 * 1024 / (stride_of(m) * 4));
        const double t = std::ceil(chunks / room) * c / 32 * 0.3 + chunks * stride_of(m) * 16 / 1.5e6 + chunks / G / 16;
        if (t < best_t) {
            best_t = t;
            best = c;
        }
    }
    return best;
}

struct SortSpace {
    int32_t *table = nullptr, *total = nullptr, *val[2] = {};
    uint32_t* key[2] = {};
    int64_t bytes = 0;
    int64_t chunk = 1;
    SortSpace(void* ws, int64_t n, int G, int64_t m)
    {
        if (by_block(n, m)) return;
        Carve c(ws);
        chunk = chunk_of(n, G, m);
        const int64_t chunks = (n + chunk - 1) / chunk;
        table = c.take<int32_t>(chunks * G * stride_of(m));
        total = c.take<int32_t>((int64_t)G * stride_of(m));
        key[0] = c.take<uint32_t>(n * G);
        if (passes_of(m) > 1) {
            key[1] = c.take<uint32_t>(n * G);
            for (int i = 0; i < 2; ++i) val[i] = c.take<int32_t>(n * G);
        }
        bytes = c.used;
    }
};

}  // namespace

int64_t sort_workspace(int64_t n, int G, int64_t m) { return SortSpace(nullptr, n, G, m).bytes; }

cudaError_t launch_sort_indices(int64_t n, int G, int64_t m, const int32_t* idx, int32_t* order, int32_t* offset, void* ws,
                                cudaStream_t s)
{
    const Launch l{s, nullptr, nullptr, true};
    if (by_block(n, m))
        return launch_granted(s, block_sort_kernel, dim3((unsigned)G), kBlockThreads, stride_of(m) * 8 + (n + 1) / 2 * 4, (int)n, G, m, idx, order, offset);
    const SortSpace sp(ws, n, G, m);
    const int passes = passes_of(m);
    Pass p{};
    p.n = n;
    p.m = m;
    p.G = G;
    p.chunk = sp.chunk;
    p.chunks = (int)((n + p.chunk - 1) / p.chunk);
    p.bins = bins_of(m);
    p.stride = stride_of(m);
    p.mask = passes == 1 ? -1 : (1 << digit_bits(m)) - 1;
    const dim3 grid((unsigned)p.chunks, (unsigned)G);
    // pass i reads keys i & 1 (the first writes them beforehand) and leaves the other ones
    for (int i = 0; i < passes; ++i) {
        const bool last = i + 1 == passes;
        p.shift = i * digit_bits(m);
        p.idx = i == 0 ? idx : nullptr;
        p.key = sp.key[i & 1];
        p.val = i == 0 ? nullptr : sp.val[i & 1];
        p.key_out = passes == 1 ? nullptr : sp.key[(i + 1) & 1];
        p.val_out = last ? order : sp.val[(i + 1) & 1];
        cudaError_t e = p.chunks ? launch_granted(s, count_kernel, grid, 256, p.stride * 4, p, sp.table) : cudaSuccess;
        if (e == cudaSuccess)
            e = launch_kernel(l, chunk_scan_kernel, dim3((p.stride + 127) / 128, (unsigned)G), 128, 0, 1, sp.table, sp.total, p.chunks, p.stride);
        if (e == cudaSuccess)
            e = launch_kernel(l, bin_scan_kernel, dim3((unsigned)G), 1024, 0, 1, sp.total, passes == 1 ? offset : nullptr, p.bins, p.stride);
        if (e == cudaSuccess && p.chunks) e = launch_granted(s, place_kernel, grid, 128, p.stride * 4, p, sp.table, sp.total);
        if (e != cudaSuccess) return e;
    }
    if (passes > 1)
        return launch_kernel(l, bounds_kernel, dim3((unsigned)((m + 256) / 256), (unsigned)G), 256, 0, 1, sp.key[passes & 1], offset, n, m);
    return cudaSuccess;
}

}  // namespace ckv
