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

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

// One element as a word's low bits, and back, and times a gate (the product rounded once).
__device__ __forceinline__ uint32_t bits_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ uint32_t bits_of(uint16_t v) { return v; }
template <typename E>
__device__ __forceinline__ uint32_t scaled(uint32_t word, float f)
{
    if (sizeof(E) == 4) return __float_as_uint(__uint_as_float(word) * f);
    return pack_bf16(__uint_as_float(word << 16) * f, __uint_as_float(word & 0xffff0000u) * f);
}

// Lookup.  A warp takes 32 rows at a time: a lane fetches one row's index and score and works out where its pool row lies and the
// gate; then the lanes run over the rows' 4-byte words side by side, so that loads and stores move whole lines whatever the
// widths (a pool row of 60 or 62 bytes lies on no wider boundary).  log_words: words of a row, a power of two.
// WORDS: no word holds elements of both parts, and the arrays lie on words; else element by element.
template <typename E, bool WORDS>
__global__ void __launch_bounds__(256) gather_kernel(int64_t rows, int G, int log_words, int skip, int ds, int64_t m, bool store_words,
                                                     const E* __restrict__ pool, const int32_t* __restrict__ idx,
                                                     const E* __restrict__ user, const float* __restrict__ score, E* __restrict__ out)
{
    constexpr int PER = 4 / (int)sizeof(E);  // elements of a word
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * 8;
    for (int64_t r0 = (blockIdx.x * (int64_t)8 + (threadIdx.x >> 5)) * 32; r0 < rows; r0 += warps * 32) {
        const int n_rows = (int)min(rows - r0, (int64_t)32);
        int64_t from = -1;
        float gate = 1.f;
        if (lane < n_rows) {
            const int32_t j = __ldg(idx + r0 + lane);
            if (j >= 0 && j < m) from = ((r0 + lane) % G * m + j) * ds;
            if (score) gate = sigmoid(__ldg(score + r0 + lane));
        }
#pragma unroll 4
        for (int i = 0; i < 1 << log_words; ++i) {
            const int w = 32 * i + lane, k = w >> log_words, c = (w - (k << log_words)) * PER;
            const int64_t at = __shfl_sync(0xffffffffu, from, k);
            const float f = __shfl_sync(0xffffffffu, gate, k);
            if (k >= n_rows) continue;
            const E *u = user + (r0 + k) * skip + c, *p = pool + at + (c - skip);
            uint32_t v = 0;
            if (WORDS) {
                if (c < skip) v = __ldg(reinterpret_cast<const uint32_t*>(u));
                else if (at >= 0) {
                    v = __ldg(reinterpret_cast<const uint32_t*>(p));
                    if (score) v = scaled<E>(v, f);
                }
            } else {
#pragma unroll
                for (int q = 0; q < PER; ++q) {
                    uint32_t x = 0;
                    if (c + q < skip) x = bits_of(u[q]);
                    else if (at >= 0) {
                        x = bits_of(p[q]);
                        if (score) x = scaled<E>(x, f);
                    }
                    v |= PER == 2 ? (x & 0xffffu) << (16 * q) : x;
                }
            }
            E* o = out + ((r0 << log_words) + w) * PER;
            if (store_words) *reinterpret_cast<uint32_t*>(o) = v;
            else {
                const uint16_t half[2] = {(uint16_t)v, (uint16_t)(v >> 16)};
#pragma unroll
                for (int q = 0; q < 2; ++q) reinterpret_cast<uint16_t*>(o)[q] = half[q];
            }
        }
    }
}

// ---- sums over runs of equal entries ---------------------------------------------------------------------------
// The sorted positions of a group are cut into chunks of equal length, whatever the entries.  LANES lanes walk a chunk, 16 bytes of
// a row each; rows of several chunks travel at a time, kAhead of each.  Runs that lie inside the chunk are written; the one that
// began before it and the one that goes on behind it leave a partial sum (head, tail), which join_kernel adds up in the
// order of the chunks.  Nothing depends on the order in which warps run.
constexpr int kAhead = 4, kSegThreads = 128;

template <typename E>
struct Row16 {  // 16 bytes of a row
    static constexpr int N = 16 / (int)sizeof(E);
    E v[N];
};

template <typename E, int LANES>
__global__ void __launch_bounds__(kSegThreads) segment_kernel(const SegmentArgs a, float* __restrict__ part, float* __restrict__ wpart,
                                                              int32_t* __restrict__ goes_on, int chunks, int chunk, int wide)
{
    constexpr int N = Row16<E>::N, PER_BLOCK = kSegThreads / LANES;
    const int sub = threadIdx.x % LANES, g = blockIdx.y, col0 = sub * N, ds = a.width - a.skip;
    const int c = blockIdx.x * PER_BLOCK + threadIdx.x / LANES;
    const bool live = c < chunks;
    const int32_t *order = a.order + (int64_t)g * a.n, *offset = a.offset + (int64_t)g * (a.m + 1);
    const int64_t begin = live ? (int64_t)c * chunk : a.n, end = min(begin + chunk, a.n);
    // the entry of the first position: the last j with offset[j] <= begin (m: no entry)
    int64_t lo = 0, hi = live ? a.m : 0;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) / 2;
        if (__ldg(offset + mid) <= begin) lo = mid;
        else hi = mid - 1;
    }
    int64_t j = lo, run_end = !live ? a.n : j < a.m ? offset[j + 1] : a.n;
    bool head = live && offset[j] < begin;
    float acc[N] = {}, own[N] = {}, wsum = 0.f;
    const int64_t at = ((int64_t)g * chunks + c) * 2;
    auto fetch_pool = [&] {
        if (!a.pool) return;
        const E* p = (const E*)a.pool + ((int64_t)g * a.m + j) * ds + col0 - a.skip;
#pragma unroll
        for (int q = 0; q < N; ++q) own[q] = j < a.m && col0 + q >= a.skip ? widen(__ldg(p + q)) : 0.f;
    };
    auto flush = [&](bool tail) {
        if (j < a.m) {
            const bool partial = head || tail;
            float* to = partial ? part + (at + (head ? 0 : 1)) * a.width + col0 : a.sum + ((int64_t)g * a.m + j) * ds + col0 - a.skip;
            if (partial || wide == 4) {  // whole 16-byte pieces
                if (partial || col0 >= a.skip) {
#pragma unroll
                    for (int q = 0; q < N; q += 4) *reinterpret_cast<float4*>(to + q) = make_float4(acc[q], acc[q + 1], acc[q + 2], acc[q + 3]);
                }
            } else if (wide == 2) {
#pragma unroll
                for (int q = 0; q < N; q += 2)
                    if (col0 + q >= a.skip) *reinterpret_cast<float2*>(to + q) = make_float2(acc[q], acc[q + 1]);
            } else {
#pragma unroll
                for (int q = 0; q < N; ++q)
                    if (col0 + q >= a.skip) to[q] = acc[q];
            }
            if (a.weight_sum && sub == 0) {
                if (partial) wpart[at + (head ? 0 : 1)] = wsum;
                else a.weight_sum[(int64_t)g * a.m + j] = wsum;
            }
        }
#pragma unroll
        for (int q = 0; q < N; ++q) acc[q] = 0.f;
        wsum = 0.f;
        head = false;
    };
    if (live) fetch_pool();
    const int64_t last = begin + chunk;  // (chunks of a warp take as many steps each: the lanes stay together)
    for (int64_t t0 = begin; t0 < last; t0 += kAhead) {
        int32_t pos[kAhead];
        uint4 raw[kAhead];
        float sc[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            pos[k] = t0 + k < end ? __ldg(order + t0 + k) : -1;
            if (pos[k] >= a.n) pos[k] = -1;  // not an order
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const bool real = pos[k] >= 0;
            raw[k] = real ? __ldg(reinterpret_cast<const uint4*>((const E*)a.rows + pos[k] * a.stride + g * a.group_stride + col0)) : make_uint4(0, 0, 0, 0);
            sc[k] = real && a.score ? __ldg(a.score + (int64_t)pos[k] * a.G + g) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t t = t0 + k;
            if (t >= run_end && t < end) {
                flush(false);
                do {
                    ++j;
                    run_end = j < a.m ? __ldg(offset + j + 1) : a.n;
                } while (t >= run_end);
                fetch_pool();
            }
            const E* v = reinterpret_cast<const E*>(&raw[k]);
            const bool real = pos[k] >= 0;
            const float w = !real ? 0.f : !a.score ? 1.f : a.pool ? sigmoid(sc[k]) : sc[k];
            float dot = 0.f;
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const float x = widen(v[q]);
                if (real) acc[q] = fmaf(w, x, acc[q]);
                dot = fmaf(own[q], x, dot);
            }
            wsum += w;
            const int64_t o = (int64_t)pos[k] * a.G + g;
            if (a.d_user && real && col0 < a.skip) {
#pragma unroll
                for (int q = 0; q < N; ++q)
                    if (col0 + q < a.skip) ((E*)a.d_user)[o * a.skip + col0 + q] = v[q];
            }
            if (a.d_score) {
#pragma unroll
                for (int d = LANES / 2; d > 0; d /= 2) dot += __shfl_xor_sync(0xffffffffu, dot, d);
                if (sub == 0 && real) a.d_score[o] = j < a.m ? dot * w * sigmoid(-sc[k]) : 0.f;
            }
        }
    }
    if (!live) return;
    const bool tail = run_end > end;
    if (sub == 0) goes_on[(int64_t)g * chunks + c] = tail && !head && j < a.m ? (int32_t)j : -1;  // began here, ends in a later chunk
    flush(tail);
}

// Blocks of the first kind: the runs that began in chunk c and go on behind it, a warp per chunk; runs of many chunks by the whole block,
// an eighth of the chunks per warp.  Blocks of the second kind: entries without a position.
constexpr int kJoinWarps = 8, kLongRun = 16;
__global__ void __launch_bounds__(32 * kJoinWarps) join_kernel(const SegmentArgs a, const float* __restrict__ part, const float* __restrict__ wpart,
                                                               const int32_t* __restrict__ goes_on, int chunks, int chunk, int join_blocks)
{
    __shared__ float eighth[kJoinWarps][132];
    __shared__ int32_t entry[kJoinWarps], upto[kJoinWarps];
    const int g = blockIdx.y, ds = a.width - a.skip, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t* offset = a.offset + (int64_t)g * (a.m + 1);
    if ((int)blockIdx.x >= join_blocks) {
        const int64_t j0 = ((int64_t)((int)blockIdx.x - join_blocks) * kJoinWarps + warp) * 32, j = j0 + lane;
        unsigned empty = __ballot_sync(0xffffffffu, j < a.m && __ldg(offset + min(j, a.m)) == __ldg(offset + min(j + 1, a.m)));
        if (a.weight_sum && (empty >> lane & 1)) a.weight_sum[(int64_t)g * a.m + j] = 0.f;
        for (; empty; empty &= empty - 1)
            for (int c = lane; c < ds; c += 32) a.sum[((int64_t)g * a.m + j0 + __ffs(empty) - 1) * ds + c] = 0.f;
        return;
    }
    // columns lane, lane + 32, ... of the head parts of chunks [from, to), and (column `width`) of the weights
    auto add_heads = [&](int from, int to, float (&sum)[5]) {
#pragma unroll 4
        for (int k = from; k < to; ++k) {
            const float* p = part + ((int64_t)g * chunks + k) * 2 * a.width;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (lane + 32 * q < a.width) sum[q] += __ldg(p + lane + 32 * q);
            if (a.weight_sum) sum[4] += __ldg(wpart + ((int64_t)g * chunks + k) * 2);
        }
    };
    auto put = [&](int64_t j, const float (&sum)[5]) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int col = lane + 32 * q;
            if (col >= a.skip && col < a.width) a.sum[((int64_t)g * a.m + j) * ds + col - a.skip] = sum[q];
        }
        if (a.weight_sum && lane == 0) a.weight_sum[(int64_t)g * a.m + j] = sum[4];
    };
    auto tail_of = [&](int c, float (&sum)[5]) {
        const int64_t at = ((int64_t)g * chunks + c) * 2 + 1;
#pragma unroll
        for (int q = 0; q < 4; ++q) sum[q] = lane + 32 * q < a.width ? __ldg(part + at * a.width + lane + 32 * q) : 0.f;
        sum[4] = a.weight_sum ? __ldg(wpart + at) : 0.f;
    };
    const int c = blockIdx.x * kJoinWarps + warp;
    const int32_t j = c < chunks ? __ldg(goes_on + (int64_t)g * chunks + c) : -1;
    int to = 0;
    if (j >= 0) to = min((__ldg(offset + j + 1) - 1) / chunk + 1, chunks);  // behind the last chunk that holds some of it
    const bool is_long = j >= 0 && to - c > kLongRun;
    if (lane == 0) {
        entry[warp] = is_long ? j : -1;
        upto[warp] = to;
    }
    if (j >= 0 && !is_long) {
        float sum[5];
        tail_of(c, sum);
        add_heads(c + 1, to, sum);
        put(j, sum);
    }
    __syncthreads();
    for (int w = 0; w < kJoinWarps; ++w) {
        if (entry[w] < 0) continue;
        const int first = blockIdx.x * kJoinWarps + w + 1, n = upto[w] - first;
        float sum[5] = {};
        add_heads(first + (int)((int64_t)n * warp / kJoinWarps), first + (int)((int64_t)n * (warp + 1) / kJoinWarps), sum);
#pragma unroll
        for (int q = 0; q < 4; ++q) eighth[warp][lane + 32 * q] = sum[q];
        if (lane == 0) eighth[warp][128] = sum[4];
        __syncthreads();
        if (warp == w) {
            tail_of(first - 1, sum);
            for (int k = 0; k < kJoinWarps; ++k) {
#pragma unroll
                for (int q = 0; q < 4; ++q) sum[q] += eighth[k][lane + 32 * q];
                sum[4] += eighth[k][128];
            }
            put(entry[w], sum);
        }
        __syncthreads();
    }
}

// Positions of a chunk: short ones until the chunks' lanes fill the SMs, long ones to leave few partial sums.
int chunk_of(int64_t n, int G)
{
    int c = 8;
    while (c < 128 && n * G / c > 16384) c *= 2;
    return c;
}

struct SegmentSpace {
    float *part, *wpart;
    int32_t* goes_on;
    int64_t bytes;
    SegmentSpace(void* ws, int64_t n, int G, int width)
    {
        Carve c(ws);
        const int64_t chunk = chunk_of(n, G), chunks = (n + chunk - 1) / chunk;
        part = c.take<float>(chunks * G * 2 * width);
        wpart = c.take<float>(chunks * G * 2);
        goes_on = c.take<int32_t>(chunks * G);
        bytes = c.used;
    }
};

template <typename E>
cudaError_t launch_segments(const SegmentArgs& a, const SegmentSpace& sp, int chunks, int chunk, int wide, cudaStream_t s)
{
    const Launch l{s, nullptr, nullptr};
    auto go = [&](auto kernel, int lanes) {
        const int per_block = kSegThreads / lanes;
        return launch_kernel(l, kernel, dim3((unsigned)((chunks + per_block - 1) / per_block), (unsigned)a.G), kSegThreads, 0, 1, a, sp.part, sp.wpart,
                             sp.goes_on, chunks, chunk, wide);
    };
    switch (a.width * (int)sizeof(E)) {
        case 32: return go(segment_kernel<E, 2>, 2);
        case 64: return go(segment_kernel<E, 4>, 4);
        case 128: return go(segment_kernel<E, 8>, 8);
        case 256: return go(segment_kernel<E, 16>, 16);
        default: return go(segment_kernel<E, 32>, 32);
    }
}

template <typename E>
cudaError_t launch_gather_t(int64_t n, int G, int D, int ds, int64_t m, const void* pool, const int32_t* idx, const void* user,
                            const float* score, void* out, cudaStream_t s)
{
    const int skip = D - ds, per = 4 / (int)sizeof(E);
    const bool words = skip % per == 0 && (((uintptr_t)pool | (uintptr_t)user) & 3) == 0;
    int log_words = 0;
    while (per << log_words < D) ++log_words;
    const int64_t blocks = std::min<int64_t>((n * G + 255) / 256, 148 * 8);
    return launch_kernel(Launch{s, nullptr, nullptr}, words ? gather_kernel<E, true> : gather_kernel<E, false>, dim3((unsigned)blocks), 256, 0, 1, n * G, G,
                         log_words, skip, ds, m, ((uintptr_t)out & 3) == 0, (const E*)pool, idx, (const E*)user, score, (E*)out);
}

}  // namespace

cudaError_t launch_gather(int dtype, int64_t n, int G, int D, int ds, int64_t m, const void* pool, const int32_t* idx,
                          const void* user, const float* score, void* out, cudaStream_t s)
{
    return dtype == CKV_F32 ? launch_gather_t<float>(n, G, D, ds, m, pool, idx, user, score, out, s)
                            : launch_gather_t<uint16_t>(n, G, D, ds, m, pool, idx, user, score, out, s);
}

int64_t segment_workspace(int64_t n, int G, int width) { return SegmentSpace(nullptr, n, G, width).bytes; }

cudaError_t launch_segment_sum(int dtype, const SegmentArgs& a, void* ws, cudaStream_t s)
{
    const SegmentSpace sp(ws, a.n, a.G, a.width);
    const int chunk = chunk_of(a.n, a.G), chunks = (int)((a.n + chunk - 1) / chunk), ds = a.width - a.skip;
    // floats of a sum's row that can be stored at a time
    const int wide = ((uintptr_t)a.sum & 15) == 0 && ds % 4 == 0 && a.skip % (dtype == CKV_F32 ? 4 : 8) == 0 ? 4
                     : ((uintptr_t)a.sum & 7) == 0 && ds % 2 == 0 && a.skip % 2 == 0 ? 2 : 1;
    cudaError_t e = cudaSuccess;
    if (chunks > 0) e = dtype == CKV_F32 ? launch_segments<float>(a, sp, chunks, chunk, wide, s) : launch_segments<uint16_t>(a, sp, chunks, chunk, wide, s);
    const int join_blocks = (chunks + kJoinWarps - 1) / kJoinWarps, empty_blocks = (int)((a.m + 32 * kJoinWarps - 1) / (32 * kJoinWarps));
    if (e == cudaSuccess)
        e = launch_kernel(Launch{s, nullptr, nullptr}, join_kernel, dim3((unsigned)(join_blocks + empty_blocks), (unsigned)a.G), 32 * kJoinWarps, 0, 1, a, sp.part,
                          sp.wpart, sp.goes_on, chunks, chunk, join_blocks);
    return e;
}

}  // namespace ckv
