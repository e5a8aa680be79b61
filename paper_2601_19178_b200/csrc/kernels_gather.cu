// Gated lookup of pool rows (Eq. Kc, training branch) and its gradient.
//
//   out[i][g]   = (user[i][g] | s_i pool[g][I_i]),  s = sigmoid(score) or 1; a position without an entry gets zeros
//   d_pool[g][j] = sum over the positions of entry j of s_i d_out[i][g][skip:], in a fixed order of partial sums
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

// A word (two bf16 or one fp32) times a gate, each product rounded once.
template <typename E>
__device__ __forceinline__ uint32_t scaled(uint32_t word, float f)
{
    if (sizeof(E) == 4) return __float_as_uint(__uint_as_float(word) * f);
    return pack_bf16(__uint_as_float(word << 16) * f, __uint_as_float(word & 0xffff0000u) * f);
}
// 16 bytes by loads of LOAD bytes, which is what the address lies on.
template <int LOAD>
__device__ __forceinline__ void load16(uint32_t (&w)[4], const void* p)
{
    if (LOAD == 16) {
        const uint4 v = ld(reinterpret_cast<const uint4*>(p));
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else if (LOAD == 4) {
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = ld(reinterpret_cast<const uint32_t*>(p) + q);
    } else {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = ld(h + 2 * q) | (uint32_t)ld(h + 2 * q + 1) << 16;
    }
}

// Lookup.  A warp takes up to 32 rows at a time: a lane fetches one row's index and score and works out where its pool row lies and
// the gate; then the lanes run over the rows' 16-byte pieces side by side.  A pool row of 60 or 62 bytes lies on no wider
// boundary than a word or an element: LOAD is what all pieces lie on.  log_pieces: of a row; log_rows: rows of a warp, fewer
// where there are few, so that a warp's chain of loads is short.  skip: elements of a row in front of the pool's, the user's or
// (widened pool) none.  Bound by the rows written (537 MB alone take 106 us) and the L1, through which pool rows and user parts
// come (issue slots 73 % used): 1048576 x 8 rows of 64 bytes, of which 4 bytes are the user's, 158 us with the copy of the pool.  200 x 2 rows: 2.4.
// STREAMED: stores of 16 bytes that leave the L2 to the pool.
template <typename E, int LOAD, bool STREAMED>
__global__ void __launch_bounds__(256) gather_kernel(int64_t rows, int G, int log_pieces, int log_rows, int skip, int user_width, int user_bytes, int ds, int64_t m, int store,
                                                     const E* pool, const int32_t* idx,
                                                     const E* user, const float* score, E* out)
{
    constexpr int N = 16 / (int)sizeof(E), PER = 4 / (int)sizeof(E);  // elements of a piece, of a word
    const int lane = threadIdx.x & 31, bytes = (skip + ds) * (int)sizeof(E);  // skip + ds: a row of `out`
    const int64_t step = (int64_t)gridDim.x * 8 << log_rows;
    grid_dependency_wait();
    constexpr uint32_t kNone = 0xffffffffu;
    // index and score of the next rows are on their way while rows are copied
    int32_t idx_next = -1;
    float score_next = 0.f;
    auto look_ahead = [&](int64_t r0) {
        const int64_t r = r0 + lane;
        const bool there = lane < 1 << log_rows && r < rows;
        idx_next = there ? ld(idx + r) : -1;
        if (score) score_next = there ? ld(score + r) : 0.f;
    };
    int64_t r0 = (blockIdx.x * (int64_t)8 + (threadIdx.x >> 5)) << log_rows;
    int group = (int)((r0 + lane) % G);  // of the lane's row
    const int step_groups = (int)(step % G);
    look_ahead(r0);
    for (; r0 < rows; r0 += step) {
        const int n_rows = (int)min(rows - r0, (int64_t)1 << log_rows);
        const uint32_t from = idx_next >= 0 && idx_next < m ? (uint32_t)group * (uint32_t)m + (uint32_t)idx_next : kNone;  // (no pool has as many rows)
        const float gate = score ? sigmoid(score_next) : 1.f;
        look_ahead(r0 + step);
        group += step_groups - (group + step_groups >= G ? G : 0);
        char* const to = reinterpret_cast<char*>(out) + r0 * bytes;
#pragma unroll 4
        for (int i = 0; i < 1 << (log_pieces + log_rows - 5); ++i) {
            const int w = 32 * i + lane, k = w >> log_pieces, c = (w - (k << log_pieces)) * N;
            const uint32_t picked = __shfl_sync(0xffffffffu, from, k);
            const float f = __shfl_sync(0xffffffffu, gate, k);
            if (k >= n_rows) continue;
            const int64_t at = (int64_t)picked * ds;
            uint32_t v[4] = {};
            if (picked != kNone) {
                if (c >= skip) load16<LOAD>(v, pool + at + (c - skip));
                else {  // a piece with elements of both parts, or of the user's alone
#pragma unroll
                    for (int q = 0; q < N; ++q)
                        if (c + q >= skip) {
                            const E x = ld(pool + at + (c + q - skip));
                            v[q / PER] |= sizeof(E) == 2 ? (uint32_t)(uint16_t)x << (16 * (q % PER)) : __float_as_uint((float)x);
                        }
                }
                if (score)
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[q] = scaled<E>(v[q], f);
            }
            if (c < user_width) {
                const E* u = user + (r0 + k) * user_width + c;
                if (user_bytes == 4) v[0] = ld(reinterpret_cast<const uint32_t*>(u));
                else if (user_bytes == 8) {
                    const uint2 x = ld(reinterpret_cast<const uint2*>(u));
                    v[0] = x.x, v[1] = x.y;
                } else if (user_bytes == 16) load16<16>(v, u);  // whole pieces are the user's
                else if (user_bytes == 2) v[0] = (v[0] & 0xffff0000u) | ld(reinterpret_cast<const uint16_t*>(u));
                else
#pragma unroll
                for (int q = 0; q < N; ++q)
                    if (c + q < user_width) {
                        const E x = ld(u + q);
                        if (sizeof(E) == 4) v[q / PER] = __float_as_uint((float)x);
                        else v[q / PER] = (v[q / PER] & (q % PER ? 0xffffu : 0xffff0000u)) | (uint32_t)(uint16_t)x << (16 * (q % PER));
                    }
            }
            char* const o = to + w * 16;
            if (STREAMED) __stcs(reinterpret_cast<uint4*>(o), make_uint4(v[0], v[1], v[2], v[3]));
            else if (store == 16) *reinterpret_cast<uint4*>(o) = make_uint4(v[0], v[1], v[2], v[3]);
            else if (store == 4) {
#pragma unroll
                for (int q = 0; q < 4; ++q) reinterpret_cast<uint32_t*>(o)[q] = v[q];
            } else {
#pragma unroll
                for (int q = 0; q < 8; ++q) reinterpret_cast<uint16_t*>(o)[q] = (uint16_t)(v[q / 2] >> (16 * (q % 2)));
            }
        }
    }
}

// ---- sums over runs of equal entries ---------------------------------------------------------------------------
// The sorted positions of a group are cut into chunks of equal length, whatever the entries.  LANES lanes walk a chunk, 16 bytes of
// a row each.  A run that lies inside the chunk is written; the one that began before it and the one that goes on behind it leave a
// partial sum (head, tail), which the block joins in the order of its chunks, and of the blocks join_kernel.  Nothing
// depends on the order in which warps run.  1048576 x 4 rows of 128 bytes with gate, d_score and d_user: 222 us again and
// again on the same arrays, 262 on other ones each time, the bare sums some two thirds of it; neither memory (2.8 TB/s) nor issue (47 %) is full: the turns' chains of loads, shuffles and shared memory
// bind, at the 20 warps per SM that their registers and stages leave, next to three sectors per row of which a few bytes are
// wanted.  20011 x 4 rows: 13 us and the join, all latency (search of the first entry 3, rows 1, runs of few positions 4).
constexpr int kSegThreads = 128;

// sigmoid(x) and 1 - sigmoid(x)
__device__ __forceinline__ float2 sigmoids(float x)
{
    const float e = expf(-fabsf(x)), big = 1.f / (1.f + e), small = e * big;
    return x >= 0.f ? make_float2(big, small) : make_float2(small, big);
}

// <row, pool row> over the pool's columns alone.  In the lanes' products the pool's row has zeros in front of them, which a user part that is
// infinite or no number turns into NaN: a product that is not a number is taken again, by the lane that stores it.  (1048576 x 4 rows of 128
// bytes: 215 us without, 222 so, 223 with masked rows, 245 with a second look at a chunk's stores; other widths within 1 %, masked 2 to 6 %.)
template <typename E>
__device__ __noinline__ float pool_product(const E* row, const E* pool_row, int n)
{
    float sum = 0.f;
#pragma unroll 1
    for (int k = 0; k < n; ++k) sum = fmaf(widen(row[k]), widen(pool_row[k]), sum);
    return sum;
}

// The last j in [lo, hi] with offset[j] <= pos; offset[lo] <= pos.
__device__ __forceinline__ int64_t entry_of(const int32_t* offset, int64_t pos, int64_t lo, int64_t hi)
{
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) / 2;
        if (ld(offset + mid) <= pos) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}
// The same for two positions, by LANES lanes that look at as many places at a time (all lanes of the warp take part).
template <int LANES>
__device__ __forceinline__ void entries_of_group(const int32_t* offset, const int64_t (&pos)[2], uint32_t top, uint32_t (&lo)[2])
{
    const int lane = threadIdx.x & 31, sub = lane % LANES;
    const unsigned mine = (LANES == 32 ? 0xffffffffu : (1u << LANES % 32) - 1) << (lane - sub);
    uint32_t hi[2] = {top, top};
    lo[0] = lo[1] = 0;
    while (__any_sync(0xffffffffu, lo[0] < hi[0] || lo[1] < hi[1])) {
        bool below[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t left = hi[k] - lo[k], ahead = (left + LANES - 1) / LANES * (sub + 1);  // (at most 2^31 + 31)
            below[k] = left && ahead <= left && ld(offset + lo[k] + ahead) <= pos[k];
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t n = __popc(__ballot_sync(0xffffffffu, below[k]) & mine);  // places at or before the entry
            const uint32_t step = (hi[k] - lo[k] + LANES - 1) / LANES;
            lo[k] += n * step;
            hi[k] = min(hi[k], lo[k] + max(step, 1u) - 1);
        }
    }
}

// Each of LANES lanes has its share of AHEAD rows' sums: added up so that row sub + i LANES ends in dot[i] of lane `sub`.  With every step a
// lane gives away the rows that are not its own.
template <int LANES, int AHEAD>
__device__ __forceinline__ void share_out(float (&dot)[AHEAD], int sub)
{
    if constexpr (LANES >= AHEAD) {
#pragma unroll
        for (int d = LANES / 2; d >= AHEAD; d /= 2)
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) dot[k] += __shfl_xor_sync(0xffffffffu, dot[k], d);
#pragma unroll
        for (int half = AHEAD / 2; half > 0; half /= 2)
#pragma unroll
            for (int k = 0; k < half; ++k) {
                const bool up = sub & half;
                const float give = up ? dot[k] : dot[k + half], keep = up ? dot[k + half] : dot[k];
                dot[k] = keep + __shfl_xor_sync(0xffffffffu, give, half);
            }
    } else {
        static_assert(LANES == 2, "a lane keeps every second row");
#pragma unroll
        for (int i = 0; i < AHEAD / 2; ++i) {
            const bool up = sub & 1;
            const float give = up ? dot[2 * i] : dot[2 * i + 1], keep = up ? dot[2 * i + 1] : dot[2 * i];
            dot[i] = keep + __shfl_xor_sync(0xffffffffu, give, 1);
        }
    }
}

// A run of rows added up by a warp.  GATED: pool is given, so that the weight is a sigmoid and d_score is wanted.
template <typename E, int LANES, bool GATED>
struct Run {
    static constexpr int N = 16 / (int)sizeof(E), SIDE = 32 / LANES, AHEAD = LANES < 8 ? LANES : 8;  // elements of a lane, rows side by side, rows of a lane
    static constexpr int ROWS = AHEAD * SIDE, WIDTH = LANES * N;
    const SegmentArgs& a;
    const int g, lane = threadIdx.x & 31, sub = lane % LANES, side = lane / LANES, col0 = sub * N;
    const int32_t* const order;
    const E* const rows;
    const int user_bytes;  // of a row's part, if one store takes it
    float acc[N], own[N], wsum;

    __device__ __forceinline__ Run(const SegmentArgs& args, int group)
        : a(args), g(group), order(args.order + (int64_t)group * args.n), rows((const E*)args.rows + group * args.group_stride + col0),
          user_bytes(args.skip <= N && ((uintptr_t)args.d_user & (args.skip * sizeof(E) - 1)) == 0 ? args.skip * (int)sizeof(E) : 0)
    {
    }
    __device__ __forceinline__ int32_t position(int64_t t, int64_t to) const
    {
        const int32_t p = lane < ROWS && t + lane < to ? ld(order + t + lane) : -1;
        return p < a.n ? p : -1;  // (not an order)
    }
    // Adds positions [from, to) of entry j (m: no entry; their user parts are copied, and their d_score is zero).
    __device__ __forceinline__ void add(int64_t from, int64_t to, int64_t j)
    {
#pragma unroll
        for (int q = 0; q < N; ++q) acc[q] = 0.f;
        wsum = 0.f;
        int32_t next = position(from, to);
        if (GATED) {
            const E* p = (const E*)a.pool + ((int64_t)g * a.m + j) * (WIDTH - a.skip) + col0 - a.skip;
#pragma unroll
            for (int q = 0; q < N; ++q) own[q] = j < a.m && col0 + q >= a.skip ? widen(ld(p + q)) : 0.f;
        }
        for (int64_t t = from; t < to; t += ROWS) {
            const int32_t pos = next;
            const int n_rows = (int)min(to - t, (int64_t)ROWS);
            const float sc = pos >= 0 && a.score ? ld(a.score + (int64_t)pos * a.G + g) : 0.f;
            uint4 raw[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (k * SIDE >= n_rows) break;
                const int32_t p = __shfl_sync(0xffffffffu, pos, k * SIDE + side);
                raw[k] = p >= 0 ? __ldcs(reinterpret_cast<const uint4*>(rows + p * a.stride)) : make_uint4(0, 0, 0, 0);  // (read once)
            }
            next = position(t + ROWS, to);
            const float2 gate = pos < 0 ? make_float2(0.f, 0.f) : !a.score ? make_float2(1.f, 0.f) : GATED ? sigmoids(sc) : make_float2(sc, 0.f);
            float dot[AHEAD] = {};
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (k * SIDE >= n_rows) break;
                const float w = __shfl_sync(0xffffffffu, gate.x, k * SIDE + side);
                const E* v = reinterpret_cast<const E*>(&raw[k]);
#pragma unroll
                for (int q = 0; q < N; ++q) {
                    const float x = widen(v[q]);
                    acc[q] = fmaf(w, x, acc[q]);
                    if (GATED) dot[k] = fmaf(own[q], x, dot[k]);
                }
                if (a.d_user) {
                    const int32_t p = __shfl_sync(0xffffffffu, pos, k * SIDE + side);
                    if (p >= 0 && col0 < a.skip) {
                        E* to_user = (E*)a.d_user + ((int64_t)p * a.G + g) * a.skip + col0;
                        if (user_bytes == 2) *reinterpret_cast<uint16_t*>(to_user) = (uint16_t)raw[k].x;
                        else if (user_bytes == 4) *reinterpret_cast<uint32_t*>(to_user) = raw[k].x;
                        else if (user_bytes == 8) *reinterpret_cast<uint2*>(to_user) = make_uint2(raw[k].x, raw[k].y);
                        else
#pragma unroll
                            for (int q = 0; q < N; ++q)
                                if (col0 + q < a.skip) to_user[q] = v[q];
                    }
                }
            }
            wsum += gate.x;  // a lane's own rows
            if (GATED && a.d_score) {
                share_out<LANES, AHEAD>(dot, sub);  // row (sub % AHEAD) SIDE + side
                const int r = sub % AHEAD * SIDE + side;
                const int32_t p = __shfl_sync(0xffffffffu, pos, r);
                const float w = __shfl_sync(0xffffffffu, gate.x, r), less = __shfl_sync(0xffffffffu, gate.y, r);
                if (p >= 0 && sub < AHEAD) {
                    float product = dot[0];
                    if (product != product && a.skip && j < a.m)
                        product = pool_product(rows - col0 + p * a.stride + a.skip, (const E*)a.pool + ((int64_t)g * a.m + j) * (WIDTH - a.skip), WIDTH - a.skip);
                    a.d_score[(int64_t)p * a.G + g] = j < a.m ? product * w * less : 0.f;
                }
            }
        }
    }
    // The sums of the whole warp, in every lane that holds their columns.
    __device__ __forceinline__ void finish()
    {
#pragma unroll
        for (int d = LANES; d < 32; d *= 2)
#pragma unroll
            for (int q = 0; q < N; ++q) acc[q] += __shfl_xor_sync(0xffffffffu, acc[q], d);
        if (!GATED && a.weight_sum)
#pragma unroll
            for (int d = 1; d < 32; d *= 2) wsum += __shfl_xor_sync(0xffffffffu, wsum, d);
    }
    __device__ __forceinline__ void put(int64_t j, int wide) const  // an entry's sums
    {
        float* to = a.sum + ((int64_t)g * a.m + j) * (WIDTH - a.skip) + col0 - a.skip;
        if (side == 0) {
            if (wide == 4) {
                if (col0 >= a.skip)
#pragma unroll
                    for (int q = 0; q < N; q += 4) *reinterpret_cast<float4*>(to + q) = make_float4(acc[q], acc[q + 1], acc[q + 2], acc[q + 3]);
            } else if (wide == 2) {
#pragma unroll
                for (int q = 0; q < N; q += 2)
                    if (col0 + q >= a.skip) *reinterpret_cast<float2*>(to + q) = make_float2(acc[q], acc[q + 1]);
            } else {
#pragma unroll
                for (int q = 0; q < N; ++q)
                    if (col0 + q >= a.skip) to[q] = acc[q];
            }
        }
        if (a.weight_sum && lane == 0) a.weight_sum[(int64_t)g * a.m + j] = wsum;
    }
};

// Few positions: a warp to each entry, which loops over its run, and one to every 32 positions without an entry (behind `entry_blocks`).  Next to
// the kernel for many it saves the search for a chunk's entries, the joins and a launch: 200 positions x 1024 entries x 2 groups 3.2 us
// and 10 + 6.
template <typename E, int LANES, bool GATED>
__global__ void __launch_bounds__(kSegThreads) few_kernel(const SegmentArgs a, int entry_blocks, int wide)
{
    const int g = blockIdx.y, warp = threadIdx.x >> 5;
    const int32_t* offset = a.offset + (int64_t)g * (a.m + 1);
    Run<E, LANES, GATED> run(a, g);
    grid_dependency_wait();
    if ((int)blockIdx.x < entry_blocks) {
        const int64_t j = (int64_t)blockIdx.x * (kSegThreads / 32) + warp;
        if (j >= a.m) return;
        const int64_t from = ld(offset + j), to = ld(offset + j + 1);
        run.add(from, from >= 0 && to <= a.n ? to : from, j);  // (else these are no offsets)
        run.finish();
        run.put(j, wide);
        return;
    }
    const int64_t from = max((int64_t)ld(offset + a.m), (int64_t)0) + ((int64_t)((int)blockIdx.x - entry_blocks) * (kSegThreads / 32) + warp) * 32;
    run.add(from, min(from + 32, a.n), a.m);
}
constexpr int64_t kFewPositions = 512;

// What a chunk leaves for its block.
struct Ends {
    int32_t head, tail;  // entries of the run that began before the chunk, and of the one that began in it and goes on; -1: none
    bool open;           // the head run goes on behind the chunk
};

// GATED: pool is given, so that the weight is a sigmoid and d_score is wanted.
template <typename E, int LANES, bool GATED>
__global__ void __launch_bounds__(kSegThreads, GATED ? 5 : 6) segment_kernel(const SegmentArgs a, float* part, float* wpart,
                                                                              int32_t* goes_on, int chunk, int wide)
{
    constexpr int N = 16 / (int)sizeof(E), GROUPS = kSegThreads / LANES;  // elements of a lane, chunks of a block
    constexpr int AHEAD = LANES < 8 ? 4 : 8, PER = AHEAD > LANES ? AHEAD / LANES : 1;  // rows on their way, looked up by a lane
    constexpr int WIDTH = LANES * N;
    __shared__ __align__(16) float ends[GROUPS][2][WIDTH];
    __shared__ float wends[GROUPS][2];
    __shared__ Ends info[GROUPS];
    __shared__ __align__(16) uint4 stage[2][AHEAD][kSegThreads];  // a turn's rows, and the next turn's on their way
    const int lane = threadIdx.x & 31, sub = lane % LANES, grp = threadIdx.x / LANES, g = blockIdx.y, col0 = sub * N, ds = WIDTH - a.skip;
    const unsigned mine = (LANES == 32 ? 0xffffffffu : (1u << LANES % 32) - 1) << (lane - sub);
    const int32_t *order = a.order + (int64_t)g * a.n, *offset = a.offset + (int64_t)g * (a.m + 1);
    const int64_t begin = min(((int64_t)blockIdx.x * GROUPS + grp) * chunk, a.n), end = min(begin + chunk, a.n);
    const bool live = begin < end;
    grid_dependency_wait();
    // a lane's share of the next rows: position of row `sub` (and `sub` + LANES)
    int32_t ahead[PER];
    auto look_ahead = [&](int64_t t0) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int64_t t = t0 + sub + i * LANES;
            ahead[i] = sub + i * LANES < AHEAD && t < end ? ld(order + t) : -1;
        }
    };
    const E* const rows = (const E*)a.rows + g * a.group_stride + col0;
    int32_t pos[PER];
    float sc[PER];
    uint64_t once;  // rows are read once, and leave the L2 to scores and results by position, of whose sectors a warp has a few bytes each
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(once));
    // rows and scores of the positions looked up, by asynchronous copies of a lane's 16 bytes of each row; then the next positions
    auto fetch_rows = [&](int buf, int64_t next) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            pos[i] = ahead[i] < a.n ? ahead[i] : -1;  // (not an order)
            sc[i] = pos[i] >= 0 && a.score ? ld(a.score + (int64_t)pos[i] * a.G + g) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int32_t p = __shfl_sync(0xffffffffu, pos[k / LANES], k % LANES, LANES);
            if (p >= 0)
                asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(smem_u32(&stage[buf][k][threadIdx.x])), "l"(rows + p * a.stride), "l"(once)
                             : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        look_ahead(next);
    };
    look_ahead(begin);
    fetch_rows(0, begin + AHEAD);
    // the entries of the first and the last position (m: no entry)
    uint32_t ends_at[2];
    entries_of_group<LANES>(offset, {begin, end - 1}, live ? (uint32_t)a.m : 0, ends_at);
    int64_t j = ends_at[0];
    const int64_t j_last = ends_at[1];
    int64_t run_end = live && j < a.m ? offset[j + 1] : a.n;
    bool head = live && offset[j] < begin;
    if (sub == 0) info[grp] = Ends{-1, -1, false};
    float acc[N] = {}, own[N] = {}, wsum = 0.f;
    auto fetch_pool = [&] {
        if (!GATED) return;
        const E* p = (const E*)a.pool + ((int64_t)g * a.m + j) * ds + col0 - a.skip;
#pragma unroll
        for (int q = 0; q < N; ++q) own[q] = j < a.m && col0 + q >= a.skip ? widen(ld(p + q)) : 0.f;
    };
    auto flush = [&](bool tail) {
        if (j < a.m) {
            if (head || tail) {
                if (sub == 0) {
                    if (head) info[grp].head = (int32_t)j, info[grp].open = tail;
                    else info[grp].tail = (int32_t)j;
                    wends[grp][head ? 0 : 1] = wsum;
                }
                float* to = &ends[grp][head ? 0 : 1][col0];
#pragma unroll
                for (int q = 0; q < N; q += 4) *reinterpret_cast<float4*>(to + q) = make_float4(acc[q], acc[q + 1], acc[q + 2], acc[q + 3]);
            } else {
                float* to = a.sum + ((int64_t)g * a.m + j) * ds + col0 - a.skip;
                if (wide == 4) {
                    if (col0 >= a.skip)
#pragma unroll
                        for (int q = 0; q < N; q += 4) *reinterpret_cast<float4*>(to + q) = make_float4(acc[q], acc[q + 1], acc[q + 2], acc[q + 3]);
                } else if (wide == 2) {
#pragma unroll
                    for (int q = 0; q < N; q += 2)
                        if (col0 + q >= a.skip) *reinterpret_cast<float2*>(to + q) = make_float2(acc[q], acc[q + 1]);
                } else {
#pragma unroll
                    for (int q = 0; q < N; ++q)
                        if (col0 + q >= a.skip) to[q] = acc[q];
                }
                if (a.weight_sum && sub == 0) a.weight_sum[(int64_t)g * a.m + j] = wsum;
            }
        }
#pragma unroll
        for (int q = 0; q < N; ++q) acc[q] = 0.f;
        wsum = 0.f;
        head = false;
    };
    if (live) fetch_pool();
    // A user part is copied in units that its size and address allow: one or two by the lane that has its row's position (500000 x 4 rows of 64
    // bf16, parts of 16 bytes: 140 us), more by the lanes that have pieces of it (parts of 10 bytes 171; the other way 154 and 188).
    const int user_bytes = a.skip * (int)sizeof(E), user_at = user_bytes | 16 | (int)((uintptr_t)a.d_user & 15), user_unit = user_at & -user_at;
    const bool user_by_row = a.d_user && user_bytes <= 2 * user_unit;
    int buf = 0;
    for (int64_t t0 = begin; t0 < begin + chunk; t0 += AHEAD, buf ^= 1) {  // (as many turns for every chunk: a warp's stay together)
        int32_t at[PER], key[PER];
        float2 gate[PER];  // weight of the row; GATED: and one less it
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            at[i] = pos[i];
            gate[i] = at[i] < 0 ? make_float2(0.f, 0.f) : !a.score ? make_float2(1.f, 0.f) : GATED ? sigmoids(sc[i]) : make_float2(sc[i], 0.f);
            key[i] = (int32_t)j;
        }
        fetch_rows(buf ^ 1, t0 + 2 * AHEAD);
        const bool mixed = t0 + AHEAD > run_end && j != j_last;
        if (mixed)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int64_t t = t0 + sub + i * LANES;
                key[i] = (int32_t)entry_of(offset, min(t, end - 1), j, j_last);
                if (GATED && key[i] < a.m) {  // the runs' pool rows, which are wanted one after the other
                    const E* p = (const E*)a.pool + ((int64_t)g * a.m + key[i]) * ds;
                    asm volatile("prefetch.global.L1 [%0];" ::"l"(p));
                    asm volatile("prefetch.global.L1 [%0];" ::"l"(p + ds - 1));
                }
            }
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();  // (a lane reads other lanes' pieces)
        const uint4* const raw = &stage[buf][0][threadIdx.x];
        // Run by run: all rows of the entry at hand, then the next entry's, until no chunk of the warp has more.  (A flush between any two
        // rows made code that did not fit the instruction cache.)
        float dot[AHEAD] = {};
        bool more, fresh = true;  // fresh: the chunk's run has not been added
        do {
            unsigned here[PER];  // rows of this run, bit k % LANES of word k / LANES
            int32_t next = INT32_MAX;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                here[i] = (__ballot_sync(0xffffffffu, fresh && at[i] >= 0 && key[i] == (int32_t)j) & mine) >> (lane - sub);
                if (at[i] >= 0 && key[i] > (int32_t)j) next = min(next, key[i]);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const float w = __shfl_sync(0xffffffffu, gate[k / LANES].x, k % LANES, LANES);
                if (here[k / LANES] >> (k % LANES) & 1) {
                    const uint4 row = raw[k * kSegThreads];
                    const E* v = reinterpret_cast<const E*>(&row);
                    float sum = 0.f;
#pragma unroll
                    for (int q = 0; q < N; ++q) {
                        const float x = widen(v[q]);
                        acc[q] = fmaf(w, x, acc[q]);
                        if (GATED) sum = fmaf(own[q], x, sum);
                    }
                    if (GATED) dot[k] = sum;
                    else wsum += w;
                }
            }
            more = __any_sync(0xffffffffu, mixed);
            if (!more) break;
#pragma unroll
            for (int d = LANES / 2; d > 0; d /= 2) next = min(next, __shfl_xor_sync(0xffffffffu, next, d));
            fresh = next != INT32_MAX;
            more = __any_sync(0xffffffffu, fresh);
            if (fresh) {
                flush(false);
                j = next;
                fetch_pool();
            }
        } while (more);
        if (mixed) run_end = j < a.m ? ld(offset + j + 1) : a.n;
        if (user_by_row) {  // lane `sub`: row `sub` (and `sub` + LANES)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                char* const to = reinterpret_cast<char*>(a.d_user) + ((int64_t)at[i] * a.G + g) * user_bytes;
                if (at[i] < 0) continue;
                for (int o = 0; o < user_bytes; o += user_unit) {
                    const char* const from = reinterpret_cast<const char*>(&stage[buf][sub + i * LANES][threadIdx.x - sub + o / 16]) + o % 16;
                    switch (user_unit) {
                        case 2: *reinterpret_cast<uint16_t*>(to + o) = *reinterpret_cast<const uint16_t*>(from); break;
                        case 4: *reinterpret_cast<uint32_t*>(to + o) = *reinterpret_cast<const uint32_t*>(from); break;
                        case 8: *reinterpret_cast<uint2*>(to + o) = *reinterpret_cast<const uint2*>(from); break;
                        default: *reinterpret_cast<uint4*>(to + o) = *reinterpret_cast<const uint4*>(from);
                    }
                }
            }
        } else if (a.d_user) {  // lane `sub`: its piece of every row
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int32_t p = __shfl_sync(0xffffffffu, at[k / LANES], k % LANES, LANES);
                if (p < 0 || col0 >= a.skip) continue;
                E* to = (E*)a.d_user + ((int64_t)p * a.G + g) * a.skip + col0;
                const uint4 row = raw[k * kSegThreads];
                if (user_unit == 16) *reinterpret_cast<uint4*>(to) = row;
                else
#pragma unroll
                    for (int q = 0; q < N; ++q)
                        if (col0 + q < a.skip) to[q] = reinterpret_cast<const E*>(&row)[q];
            }
        }
        if (GATED && a.d_score) {
            share_out<LANES, AHEAD>(dot, sub);
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (at[i] >= 0) {
                    float product = dot[i];
                    if (product != product && a.skip && key[i] < a.m)
                        product = pool_product(reinterpret_cast<const E*>(&stage[buf][sub + i * LANES][threadIdx.x - sub]) + a.skip,
                                               (const E*)a.pool + ((int64_t)g * a.m + key[i]) * ds, ds);
                    a.d_score[(int64_t)at[i] * a.G + g] = key[i] < a.m ? product * gate[i].x * gate[i].y : 0.f;
                }
        }
        __syncwarp();  // (the next turn's copies go where these rows are)
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (live) flush(j < a.m && run_end > end);
    __syncthreads();
    // the block's chunks in their order, a thread per column (and one for the weights)
    const int col = threadIdx.x;
    const int64_t block = (int64_t)g * gridDim.x + blockIdx.x;
    const bool weights = col == WIDTH % kSegThreads && a.weight_sum;  // (rows of 128 columns have no thread left: their first one does both)
    for (int pass = 0; pass < 2; ++pass) {
        if (pass == 0 ? col >= WIDTH : !weights) continue;
        float sum = 0.f;
        int32_t open = -1;
        bool before = false;  // the open run began before the block
        auto close = [&](int32_t e, int which) {
            if (which < 0) {
                if (pass) a.weight_sum[(int64_t)g * a.m + e] = sum;
                else if (col >= a.skip) a.sum[((int64_t)g * a.m + e) * ds + col - a.skip] = sum;
            } else if (pass) wpart[block * 2 + which] = sum;
            else part[(block * 2 + which) * WIDTH + col] = sum;
        };
        for (int c = 0; c < GROUPS; ++c) {
            const Ends e = info[c];
            if (e.head >= 0) {
                if (open < 0) before = true, sum = 0.f;
                sum += pass ? wends[c][0] : ends[c][0][col];
                open = e.head;
                if (!e.open) {
                    close(open, before ? 0 : -1);
                    open = -1;
                }
            }
            if (e.tail >= 0) {
                open = e.tail;
                before = false;
                sum = pass ? wends[c][1] : ends[c][1][col];
            }
        }
        if (open >= 0) close(open, before ? 0 : 1);
        if (pass == 0 && col == 0) goes_on[block] = open >= 0 && !before ? open : -1;  // began in this block, ends in a later one
    }
}

// `chunks` of `chunk` positions are the blocks of segment_kernel here.  Blocks of the first kind: the runs that began in chunk c and go on
// behind it, a warp per chunk; runs of many chunks by the whole block, an eighth of the chunks per warp.  Blocks of the second
// kind: entries without a position.
constexpr int kJoinWarps = 8, kLongRun = 8;
__global__ void __launch_bounds__(32 * kJoinWarps) join_kernel(const SegmentArgs a, const float* part, const float* wpart,
                                                               const int32_t* goes_on, int chunks, int chunk, int join_blocks)
{
    __shared__ float eighth[kJoinWarps][132];
    __shared__ int32_t entry[kJoinWarps], upto[kJoinWarps];
    const int g = blockIdx.y, ds = a.width - a.skip, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t* offset = a.offset + (int64_t)g * (a.m + 1);
    grid_dependency_wait();
    if ((int)blockIdx.x >= join_blocks) {
        const int64_t j0 = ((int64_t)((int)blockIdx.x - join_blocks) * kJoinWarps + warp) * 32, j = j0 + lane;
        unsigned empty = __ballot_sync(0xffffffffu, j < a.m && ld(offset + min(j, a.m)) == ld(offset + min(j + 1, a.m)));
        if (a.weight_sum && (empty >> lane & 1)) a.weight_sum[(int64_t)g * a.m + j] = 0.f;
        for (; empty; empty &= empty - 1)
            for (int c = lane; c < ds; c += 32) a.sum[((int64_t)g * a.m + j0 + __ffs(empty) - 1) * ds + c] = 0.f;
        return;
    }
    // columns lane, lane + 32, ... of the head parts of chunks [from, to), and (column `width`) of the weights
    auto add_heads = [&](int from, int to, float (&sum)[5]) {
#pragma unroll 8
        for (int k = from; k < to; ++k) {
            const float* p = part + ((int64_t)g * chunks + k) * 2 * a.width;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (lane + 32 * q < a.width) sum[q] += ld(p + lane + 32 * q);
            if (a.weight_sum) sum[4] += ld(wpart + ((int64_t)g * chunks + k) * 2);
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
        for (int q = 0; q < 4; ++q) sum[q] = lane + 32 * q < a.width ? ld(part + at * a.width + lane + 32 * q) : 0.f;
        sum[4] = a.weight_sum ? ld(wpart + at) : 0.f;
    };
    const int c = blockIdx.x * kJoinWarps + warp;
    const int32_t j = c < chunks ? ld(goes_on + (int64_t)g * chunks + c) : -1;
    int to = 0;
    if (j >= 0) to = min((ld(offset + j + 1) - 1) / chunk + 1, chunks);  // behind the last chunk that holds some of it
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

// Positions of a chunk: short ones until the chunks' lanes fill the SMs, long ones to leave few partial sums.  (1048576 x 4 positions: 234 us with
// 32, 217 with 64, 227 with 128, 266 with 256.)
int chunk_of(int64_t n, int G)
{
    int c = 8;
    while (c < 64 && n * G / c > 16384) c *= 2;
    return c;
}
// of a block: kSegThreads / lanes chunks
int64_t block_of(int64_t n, int G, int width, int elem) { return (int64_t)chunk_of(n, G) * kSegThreads * 16 / (width * elem); }

struct SegmentSpace {
    float *part, *wpart;
    int32_t* goes_on;
    int64_t bytes;
    SegmentSpace(void* ws, int64_t n, int G, int width, int elem)
    {
        if (n <= kFewPositions) {
            part = wpart = nullptr;
            goes_on = nullptr;
            bytes = 0;
            return;
        }
        Carve c(ws);
        const int64_t block = block_of(n, G, width, elem), blocks = (n + block - 1) / block;
        part = c.take<float>(blocks * G * 2 * width);
        wpart = c.take<float>(blocks * G * 2);
        goes_on = c.take<int32_t>(blocks * G);
        bytes = c.used;
    }
};

template <typename E>
cudaError_t launch_segments(const SegmentArgs& a, const SegmentSpace& sp, int blocks, int wide, cudaStream_t s)
{
    auto go = [&](auto gated, auto plain, auto few_gated, auto few_plain) {
        if (a.n <= kFewPositions) {
            const int warps = kSegThreads / 32, entry_blocks = (int)((a.m + warps - 1) / warps), others = a.d_user || a.d_score ? (int)((a.n + 32 * warps - 1) / (32 * warps)) : 0;
            return launch_kernel(Launch{s, nullptr, nullptr, true}, a.pool ? few_gated : few_plain, dim3((unsigned)(entry_blocks + others), (unsigned)a.G), kSegThreads, 0, 1,
                                 a, entry_blocks, wide);
        }
        return launch_kernel(Launch{s, nullptr, nullptr, true}, a.pool ? gated : plain, dim3((unsigned)blocks, (unsigned)a.G), kSegThreads, 0, 1, a, sp.part,
                             sp.wpart, sp.goes_on, chunk_of(a.n, a.G), wide);
    };
    switch (a.width * (int)sizeof(E)) {
        case 32:
            if constexpr (sizeof(E) == 2) return go(segment_kernel<E, 2, true>, segment_kernel<E, 2, false>, few_kernel<E, 2, true>, few_kernel<E, 2, false>);
        case 64: return go(segment_kernel<E, 4, true>, segment_kernel<E, 4, false>, few_kernel<E, 4, true>, few_kernel<E, 4, false>);
        case 128: return go(segment_kernel<E, 8, true>, segment_kernel<E, 8, false>, few_kernel<E, 8, true>, few_kernel<E, 8, false>);
        case 256: return go(segment_kernel<E, 16, true>, segment_kernel<E, 16, false>, few_kernel<E, 16, true>, few_kernel<E, 16, false>);
        default:
            if constexpr (sizeof(E) == 4) return go(segment_kernel<E, 32, true>, segment_kernel<E, 32, false>, few_kernel<E, 32, true>, few_kernel<E, 32, false>);
            return cudaErrorInvalidValue;
    }
}

// Pool rows behind `skip` zeros, D elements each: every piece of a row then is 16 bytes on a 16-byte boundary.
template <typename E>
__global__ void __launch_bounds__(256) widen_pool_kernel(int64_t pieces, int log_pieces, int skip, int ds, const E* pool, uint4* wide)
{
    constexpr int N = 16 / (int)sizeof(E);
    const int64_t t = blockIdx.x * (int64_t)256 + threadIdx.x;
    grid_dependency_wait();
    if (t >= pieces) return;
    const int64_t r = t >> log_pieces;
    const int c = (int)(t - (r << log_pieces)) * N;
    __align__(16) E v[N];
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = c + q >= skip ? ld(pool + r * ds + (c + q - skip)) : (E)0;
    wide[t] = *reinterpret_cast<const uint4*>(v);
}

// Whether a lookup copies the pool first.  Four loads of a piece's words (eight of its elements) keep the L1 busy for longer than the row
// takes to store (1048576 x 8 rows of 64 bytes 261 us, 158 behind a copy of 3), which pays once there are some rows per entry.
bool widens(int64_t n, int D, int ds, int64_t m, int elem) { return n >= 2 * m && (ds * elem % 16 != 0 || (D - ds) * elem % 16 != 0); }

template <typename E>
cudaError_t launch_gather_t(int64_t n, int G, int D, int ds, int64_t m, const void* pool, const int32_t* idx, const void* user,
                            const float* score, void* out, void* ws, cudaStream_t s)
{
    constexpr int e = (int)sizeof(E);
    int skip = D - ds, user_width = skip;
    int log_pieces = 0, log_rows = 5;
    while (16 << log_pieces < D * e) ++log_pieces;
    if (widens(n, D, ds, m, e)) {
        const int64_t pieces = G * m << log_pieces;
        const cudaError_t er = launch_kernel(Launch{s, nullptr, nullptr, true}, widen_pool_kernel<E>, dim3((unsigned)((pieces + 255) / 256)), 256, 0, 1, pieces,
                                             log_pieces, skip, ds, (const E*)pool, (uint4*)ws);
        if (er != cudaSuccess) return er;
        pool = ws;
        skip = 0;
        ds = D;
    }
    auto lies_on = [](const void* p, int step) { return ((uintptr_t)p | (uintptr_t)step) % 16 == 0 ? 16 : ((uintptr_t)p | (uintptr_t)step) % 4 == 0 ? 4 : 2; };
    // a user part that one load takes, or pieces that one load each takes
    const int ub = user_width * e % 16 == 0 ? 16 : user_width * e, user_bytes = (ub == 2 || ub == 4 || ub == 8 || ub == 16) && (uintptr_t)user % ub == 0 ? ub : 0;
    // A pool that takes a good part of the L2 keeps it better when the rows written leave first (300000 x 4 rows, pool of 146 MB: 90 us and 81; of
    // 29 MB: 87 and 82); a small one is there anyway (1048576 x 8 rows, 2 MB: 160 and 161).
    const int load = std::min(lies_on(pool, ds * e), lies_on(nullptr, skip * e)), store = lies_on(out, 16);
    const bool streamed = store == 16 && G * m * ds * e >= 8 << 20;
    while (log_pieces + log_rows > 5 && log_rows > 0 && (n * G >> log_rows) < 148 * 32) --log_rows;
    const int64_t per_block = (int64_t)8 << log_rows, blocks = std::min<int64_t>((n * G + per_block - 1) / per_block, 148 * 8);
    auto go = [&](auto kernel) {
        return launch_kernel(Launch{s, nullptr, nullptr, true}, kernel, dim3((unsigned)blocks), 256, 0, 1, n * G, G, log_pieces, log_rows, skip, user_width, user_bytes, ds, m, store,
                             (const E*)pool, idx, (const E*)user, score, (E*)out);
    };
    if constexpr (e == 2)
        if (load == 2) return streamed ? go(gather_kernel<E, 2, true>) : go(gather_kernel<E, 2, false>);
    if (load == 4) return streamed ? go(gather_kernel<E, 4, true>) : go(gather_kernel<E, 4, false>);
    return streamed ? go(gather_kernel<E, 16, true>) : go(gather_kernel<E, 16, false>);
}

}  // namespace

int64_t gather_workspace(int dtype, int64_t n, int G, int D, int ds, int64_t m)
{
    const int elem = dtype == CKV_F32 ? 4 : 2;
    return widens(n, D, ds, m, elem) ? G * m * D * elem : 0;
}

cudaError_t launch_gather(int dtype, int64_t n, int G, int D, int ds, int64_t m, const void* pool, const int32_t* idx,
                          const void* user, const float* score, void* out, void* ws, cudaStream_t s)
{
    return dtype == CKV_F32 ? launch_gather_t<float>(n, G, D, ds, m, pool, idx, user, score, out, ws, s)
                            : launch_gather_t<uint16_t>(n, G, D, ds, m, pool, idx, user, score, out, ws, s);
}

int64_t segment_workspace(int64_t n, int G, int width)  // of either type: the longer blocks are those of 16-bit elements
{
    return std::max(SegmentSpace(nullptr, n, G, width, 2).bytes, SegmentSpace(nullptr, n, G, width, 4).bytes);
}

cudaError_t launch_segment_sum(int dtype, const SegmentArgs& a, void* ws, cudaStream_t s)
{
    const int elem = dtype == CKV_F32 ? 4 : 2, ds = a.width - a.skip;
    const SegmentSpace sp(ws, a.n, a.G, a.width, elem);
    const int64_t block = block_of(a.n, a.G, a.width, elem);
    const int blocks = (int)((a.n + block - 1) / block);
    // floats of a sum's row that can be stored at a time
    const int wide = ((uintptr_t)a.sum & 15) == 0 && ds % 4 == 0 && a.skip % (16 / elem) == 0 ? 4
                     : ((uintptr_t)a.sum & 7) == 0 && ds % 2 == 0 && a.skip % 2 == 0 ? 2 : 1;
    cudaError_t e = cudaSuccess;
    e = dtype == CKV_F32 ? launch_segments<float>(a, sp, blocks, wide, s) : launch_segments<uint16_t>(a, sp, blocks, wide, s);
    if (a.n <= kFewPositions) return e;
    const int join_blocks = (blocks + kJoinWarps - 1) / kJoinWarps, empty_blocks = (int)((a.m + 32 * kJoinWarps - 1) / (32 * kJoinWarps));
    if (e == cudaSuccess)
        e = launch_kernel(Launch{s, nullptr, nullptr, true}, join_kernel, dim3((unsigned)(join_blocks + empty_blocks), (unsigned)a.G), 32 * kJoinWarps, 0, 1, a,
                          sp.part, sp.wpart, sp.goes_on, blocks, (int)block, join_blocks);
    return e;
}

}  // namespace ckv
