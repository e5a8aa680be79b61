// The passes of the router losses over the score matrix, on the tcgen05 tensor cores (kernels_route_loss.cu has the formulas).
//
// One side's rows stand: 128 to a block, a thread each (TMEM lane), their inputs as an A operand in TMEM.  The other side's stream
// through a ring of shared-memory stages, as B operand (a swizzled TMA box per 64 inputs).  What a streaming row adds to all its
// scores (an entry's bias, a position's -lse) comes in with the product, as one more step of K = 16: ones times the number
// cut into three bf16 parts, whose sum is the fp32 number exactly.  (Read beside the scores it cost a thread one 16-byte
// load of shared memory per four columns, whose 512 bytes take the data path four clocks, and an addition.)  A standing row's number comes
// in the same way, by a step of its own, its parts times ones: first the bias, so that every pass has the same bits for x W + b however large b
// is, then -lse.  A tile of
// scores appears in TMEM, its thread reads its row of it, and:
//   sweep_kernel (LSE, MEAN, R)  keeps a running sum.  Three blocks per CTA, two accumulators of 64 columns each (one of 96 at d_in = 128).
//   grad_kernel (DX, DW)         turns it into weights T (bf16, over the head of the scores they came from), which multiply the
//                                same tile once more, now as MN-major operand:  O += T tile.  Two blocks per CTA (one at d_in =
//                                128), each with two score buffers whose turns belong to four warps each.
// Bound by the special-function unit, 16 exponentials per clock and SM, and the FMA pipe, which takes its share of them: 32768 positions x 16384
// entries x 4 groups (2.1e9 scores, whose exponentials would take that unit alone 477 us per pass), d_in = 64: LSE 503 us, MEAN 467, R 528
// to 545, DX and DW 1300 to 1355; special-function unit 66 to 76 % busy, issue slots 57 to 65 %, tensor cores 32 to 48 %.
// Every wait is bounded: a time-out raises the CTA's abort flag, which ends all others; the CTA waits for its copies and
// products in flight, frees its TMEM, and its results are NaN.
#include <cuda_bf16.h>
#include <math_constants.h>

#include <algorithm>

#include "fit.h"
#include "ptx_helpers.cuh"
#include "tensor_map.h"

namespace ckv {
namespace {

// LSE, MEAN, R: three blocks of standing rows per CTA, four reading warps and an issuing one each, and a loading warp
constexpr int kBlocks = 3, kRows = 128 * kBlocks;
static_assert(kRows == kSweepPad, "a standing block is one of the blocks that the arrays are padded to");
constexpr int kReadWarps = 4 * kBlocks, kIssueWarp = kReadWarps, kLoadWarp = kIssueWarp + kBlocks;
constexpr int kSweepThreads = (kLoadWarp + 1) * 32;
constexpr int kStages = 6;

constexpr uint32_t kSpin = 1u << 18, kSuspend = 4000;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(kSuspend)
        : "memory");
    return ok != 0;
}
// By all lanes of a warp: waits for the phase; false when the wait ran out or another one has.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag)
{
    bool ok = bar_test(bar, parity);
    for (uint32_t i = 0; !ok && i < kSpin; ++i) {
        ok = bar_test(bar, parity);
        if ((i & 31u) == 31u && *abort_flag) break;
    }
    ok = __all_sync(0xffffffffu, ok);
    if (!ok) *abort_flag = 1;
    return ok;
}
// Named barriers of a score buffer, for the four warps whose turn it is and its block's issuing warp: "the weights of tile t stand".
// The former arrive and run on, the latter waits; once a wait has run out, a warp takes part as the issuing warp does, tile by
// tile, so that the others never wait for good.  Two in turn per buffer: who gives up on the buffer's next tile has arrived for
// this one already, and on the same barrier would count for the issuing warp.  (As mbarriers they cost some 300 clocks more each turn.)
__device__ __forceinline__ int weights_barrier(int buffer, int tile) { return 2 + 2 * buffer + ((tile >> 1) & 1); }
__device__ __forceinline__ void weights_arrive(int buffer, int tile) { asm volatile("bar.arrive %0, 160;" ::"r"(weights_barrier(buffer, tile)) : "memory"); }
__device__ __forceinline__ void weights_sync(int buffer, int tile) { asm volatile("bar.sync %0, 160;" ::"r"(weights_barrier(buffer, tile)) : "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit_to(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(acc)
        : "memory");
}
// instruction descriptor, kind::f16: fp32 accumulate, bf16 A and B, A K-major
__host__ __device__ constexpr uint32_t idesc_bf16(int M, int N, bool b_mn_major)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// A tile of rows of ROWB bytes as a TMA box with a swizzle of that span writes it, groups of eight rows ROWB * 8 bytes apart: as K-major
// operand (rows are N) and as MN-major operand (rows are K) alike.
template <int ROWB>
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr)
{
    constexpr uint64_t layout = ROWB == 128 ? 2 : 4;  // 128-byte / 64-byte swizzle
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (1ull << 16) | ((uint64_t)(ROWB * 8 >> 4) << 32) | (1ull << 46) | (layout << 61);
}
// That step's B operand: 16 bf16 per row, in groups of eight rows of 16 bytes, no swizzle (put_step of fit.h).
__device__ __forceinline__ uint64_t step_desc(uint32_t addr)
{
    return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(128 >> 4) << 16) | ((uint64_t)(256 >> 4) << 32) | (1ull << 46);
}
__device__ __forceinline__ void ld32(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,"
        "%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
// Waits for this thread's loads; the registers are operands so that nothing reads them earlier.
__device__ __forceinline__ void wait_ld32(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]),
                   "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]),
                   "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]),
                   "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}
// 16 consecutive columns of this thread's lane
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t* r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
            taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void st8(uint32_t taddr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
// A operand of the step that adds a streaming row's own number: three ones for the number's three parts.
__device__ __forceinline__ void store_ones(uint32_t taddr)
{
    const uint32_t ones[8] = {0x3f803f80u, 0x00003f80u, 0, 0, 0, 0, 0, 0};
    st8(taddr, ones);
}
// And of the one that adds a standing row's, whose B operand are `rows` rows of ones in shared memory, which the whole block writes.
__device__ __forceinline__ void store_parts(uint32_t taddr, float v)
{
    const uint2 parts = bf16_parts(v);
    const uint32_t w[8] = {parts.x, parts.y, 0, 0, 0, 0, 0, 0};
    st8(taddr, w);
}
__device__ __forceinline__ void put_ones(unsigned char* to, int rows)
{
    for (int k = threadIdx.x; k < 2 * rows; k += blockDim.x)  // groups of eight rows: their first halves, their second ones
        reinterpret_cast<uint4*>(to)[k] = k & 8 ? make_uint4(0, 0, 0, 0) : make_uint4(0x3f803f80u, 0x00003f80u, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int col, int row, int group, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(col), "r"(row), "r"(group), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void load_bytes(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}

// Two fp32 operations in one instruction.
struct F2 {
    float x, y;
};
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c)
{
    F2 d;
    asm("{\n.reg .b64 ra, rb, rc, rd;\nmov.b64 ra, {%2, %3};\nmov.b64 rb, {%4, %5};\nmov.b64 rc, {%6, %7};\n"
        "fma.rn.f32x2 rd, ra, rb, rc;\nmov.b64 {%0, %1}, rd;\n}\n"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b)
{
    F2 d;
    asm("{\n.reg .b64 ra, rb, rd;\nmov.b64 ra, {%2, %3};\nmov.b64 rb, {%4, %5};\nadd.rn.f32x2 rd, ra, rb;\nmov.b64 {%0, %1}, rd;\n}\n"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b)
{
    F2 d;
    asm("{\n.reg .b64 ra, rb, rd;\nmov.b64 ra, {%2, %3};\nmov.b64 rb, {%4, %5};\nmul.rn.f32x2 rd, ra, rb;\nmov.b64 {%0, %1}, rd;\n}\n"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float max3f(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ F2 pair(const uint32_t (&v)[32], int e) { return {__uint_as_float(v[e]), __uint_as_float(v[e + 1])}; }
__device__ __forceinline__ F2 both(float v) { return {v, v}; }
__device__ __forceinline__ F2 neg(F2 v) { return {-v.x, -v.y}; }

// 2^x on the FMA pipe, for as many of the weights as balance it with the special-function unit: x = n + f with n the nearest whole
// number, 2^f on [-1/2, 1/2] by the polynomial of degree DEG whose largest relative error is smallest (7.5e-5, 2.7e-6, 9.4e-8 for degrees 3 to 5
// with coefficients of 32 bits; the last one's constant is fixed at 1, and the others are rounded one after the other from the lowest, each fitted
// anew: its error is -1.7e-8 on average, where coefficients rounded all at once gave 5.3e-8 and 1.6e-7 at most), 2^n by its exponent bits, which the
// sum that rounds x leaves in its low bits.  Arguments are at most 0 but for rounding, and 32 where scores are 2^29 (kCoarse); below -127 the
// result is zero, and not a number stays that.
template <int DEG>
struct Exp2 {
    F2 p, scale;  // 2^x = p * scale
    __device__ __forceinline__ explicit Exp2(F2 x)
    {
        constexpr float kRound = 12582912.f + 127.f;  // 1.5 * 2^23 + 127
        asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(x.x));  // -127
        asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(x.y));
        const F2 t = add2(x, both(kRound)), f = add2(x, neg(add2(t, both(-kRound))));
        if (DEG == 3) p = fma2(fma2(fma2(both(0.0551716685f), f, both(0.242611125f)), f, both(0.693260968f)), f, both(0.999928057f));
        else if (DEG == 4)
            p = fma2(fma2(fma2(fma2(both(0.00957010221f), f, both(0.0559178591f)), f, both(0.240247443f)), f, both(0.693121791f)), f, both(0.999999285f));
        else
            p = fma2(fma2(fma2(fma2(fma2(both(0.00132539868f), f, both(0.00967128575f)), f, both(0.0555077344f)), f, both(0.240222469f)), f, both(0.693146944f)), f,
                     both(1.0f));
        scale = {__uint_as_float(__float_as_uint(t.x) << 23), __uint_as_float(__float_as_uint(t.y) << 23)};
    }
};

// Pairs of sixteen whose exponentials run on the FMA pipe, spread over them.  32768 positions x 16384 entries x 4 groups, us, with none: LSE 589,
// MEAN 572, R 582, DX 633, DW 675; with 3, 4, 5 and 6 of them: LSE 520 514 503 521, MEAN 493 478 468 481, R 547 536 543 541, DX and DW in
// one launch 1325 1330 1412 1420 (alone, DX 599 612 628 634 and DW 644 646 681 713).
constexpr int kFmaLse = 5, kFmaMean = 5, kFmaR = 4, kFmaGrad = 3;
__device__ __forceinline__ constexpr bool on_fma(int q, int of16) { return (q + 1) * of16 / 16 > q * of16 / 16; }
template <bool DW>
__device__ __forceinline__ F2 weight(F2 u, bool fma)
{
    if (!fma) return {ex2(u.x), ex2(u.y)};
    const Exp2<DW ? 4 : 3> p(u);
    return mul2(p.p, p.scale);
}

// The exponent of a weight is s log2(e) - c with c = lse log2(e) rounded once, which is off by as much as lse is as an fp32 number: at 10^6 a weight by a
// thirtieth, at 10^7 by most of itself, at 10^10 by its whole range.  MEAN, R and DW have the difference s - lse from the tensor core, where it is exact if small.  LSE, whose c is top
// log2(e), takes its residue top log2(e) - c, which one fused operation gives exactly, out of the sum.  DX takes the difference first where lse is far from zero: a branch per 32 scores, which few rows take.
constexpr float kFar = 1024.f;
__device__ __forceinline__ bool is_far(float reference) { return fabsf(reference) > kFar && reference > -CUDART_INF_F; }
__device__ __forceinline__ void move(uint32_t (&v)[32], float by)
{
#pragma unroll
    for (int q = 0; q < 32; ++q) v[q] = __float_as_uint(__uint_as_float(v[q]) + by);
}
// (Residues of references that were given up differ by no more than such scores' own rounding; with f = 2^(c - c before), which keeps them alike,
// the pass took 519 us instead of 509.)  From this `top` on, where the residue would be more than 32, lse is `top`: numbers lie 64 apart, which no
// count of equal scores moves.
constexpr float kCoarse = 536870912.f;

// A sum of many parts: what an addition loses is added with the next part.
struct LongSum {
    float s = 0.f, lost = 0.f;
    __device__ __forceinline__ void add(float v)
    {
        const float y = v - lost, t = s + y;
        lost = (t - s) - y;
        s = t;
    }
};

// ---- LSE, MEAN, R: joining the partial results of the blocks that shared a standing block's streaming rows, in the order of those blocks: by
// the one of them that is done last where all run at a time, else in a launch of its own.  (200 positions x 1024 entries x 2
// groups, both losses: 23 us and 28; 32768 x 16384 x 4, in seven rounds of blocks that each wait for their stores: 1030 and 984.)

// Every thread's results stand in memory: true in the block that is the last of n_blocks to say so.
__device__ __forceinline__ bool last_of(unsigned* ticket, unsigned n_blocks)
{
    __shared__ bool last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(ticket, 1u) + 1 == n_blocks;
    __syncthreads();
    __threadfence();
    return last;
}
// Sums over the threads of a block, in a fixed order.
template <int N>
__device__ __forceinline__ void block_sum(double (&v)[N])
{
    __shared__ double part[N][kSweepThreads / 32];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
        for (int d = 16; d > 0; d /= 2) v[k] += __shfl_xor_sync(0xffffffffu, v[k], d);
        if ((threadIdx.x & 31) == 0) part[k][threadIdx.x >> 5] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        v[k] = 0;
#pragma unroll
        for (int w = 0; w < kSweepThreads / 32; ++w) v[k] += part[k][w];
    }
}

// lse of position row0 + thread (the first kSweepPad threads), and what the peak loss and the mean weights want of the block's positions.
__device__ __forceinline__ void join_lse(const SweepArgs& a, int g, int64_t row0)
{
    const int64_t i = row0 + threadIdx.x;
    const bool has_row = threadIdx.x < kSweepPad;
    const int32_t k = has_row && i < a.n ? ld(a.idx + i * a.G + g) : -1;
    const bool real = k >= 0 && k < a.m;
    float lse = 0.f, neg = -CUDART_INF_F;
    double soft[1] = {};
    if (real) {
        const float sc = ld(a.score + i * a.G + g);
        const float2* part = reinterpret_cast<const float2*>(a.part) + g * a.np + i;
        const int64_t step = a.G * a.np;
        float top = -CUDART_INF_F, sum = 0.f;
#pragma unroll 4
        for (int z = 0; z < a.splits; ++z) {
            const float2 v = __ldcg(part + z * step);
            const float both = fmaxf(top, v.x);
            sum = both > -CUDART_INF_F ? sum * expf(top - both) + v.y * expf(v.x - both) : sum + v.y;
            top = both;
        }
        sum += ld(a.spoilt + i);
        if (top == -CUDART_INF_F && sum == 0.f) lse = top;  // every entry's score is -inf: no weight anywhere
        else {
            lse = top + logf(sum);
            neg = -lse;
        }
        soft[0] = fmaxf(-sc, 0.f) + log1pf(expf(-fabsf(sc)));  // -log sigmoid(sc)
    }
    if (has_row) {
        a.nl[g * a.np + i] = neg;
        put_step(a.nl_step, g * a.np + i, neg);
        if (i < a.n) a.lse[i * a.G + g] = lse;
    }
    const int rows = __syncthreads_count(real), live = __syncthreads_count(neg != -CUDART_INF_F);
    block_sum<1>(soft);
    if (threadIdx.x == 0) {
        const int64_t at = g * (a.np / kSweepPad) + row0 / kSweepPad;
        a.rows_part[at] = rows;
        a.live_part[at] = live;
        a.peak_part[at] = soft[0];
    }
}

// The mean weight of entry row0 + thread, and in a group's last block both losses, from partial sums in the order of the blocks.
// mean log(mean m) is summed as (u log u - u + 1) / m with u = mean m: the weights sum to one, so that nothing is added, and near
// balance, where u log u and the sum's other terms cancel, each term is as small as what it stands for.  (They sum to less by
// the share of the positions that have no weight.)
__device__ __forceinline__ void join_mean(const SweepArgs& a, int g, int64_t row0)
{
    const int blocks = (int)(a.np / kSweepPad), entry_blocks = (int)(a.mp / kSweepPad);
    double of_rows[3] = {};  // positions that take part, those with a weight, peak losses
    for (int b = threadIdx.x; b < blocks; b += kSweepThreads) {
        of_rows[0] += a.rows_part[(int64_t)g * blocks + b];
        of_rows[1] += a.live_part[(int64_t)g * blocks + b];
        of_rows[2] += a.peak_part[(int64_t)g * blocks + b];
    }
    const int64_t j = row0 + threadIdx.x;
    const bool real = threadIdx.x < kSweepPad && j < a.m;
    float sum = 0.f;
    if (real)
#pragma unroll 4
        for (int z = 0; z < a.splits; ++z) sum += __ldcg(a.part + ((int64_t)z * a.G + g) * a.mp + j);
    block_sum<3>(of_rows);
    const double rows = of_rows[0];
    double balance[1] = {};
    if (real) {
        const float mean = rows > 0 ? sum * (float)(1.0 / rows) : 0.f;
        a.mean[(int64_t)g * a.m + j] = mean;
        const double u = (double)mean * (double)a.m;
        balance[0] = (u > 0 ? u * log(u) : u * 0) - u + 1;
    }
    block_sum<1>(balance);
    if (threadIdx.x == 0) a.balance_part[(int64_t)g * entry_blocks + row0 / kSweepPad] = balance[0];
    if (!last_of(a.ticket + (int64_t)a.G * entry_blocks + g, (unsigned)entry_blocks)) return;
    balance[0] = 0;
    for (int b = threadIdx.x; b < entry_blocks; b += kSweepThreads) balance[0] += __ldcg(a.balance_part + (int64_t)g * entry_blocks + b);
    block_sum<1>(balance);
    if (threadIdx.x == 0) {
        a.loss[2 * g] = rows > 0 ? (float)(balance[0] / (double)a.m + (of_rows[1] - rows) / rows) : 0.f;
        a.loss[2 * g + 1] = rows > 0 ? (float)(of_rows[2] / rows) : 0.f;
    }
}

__device__ __forceinline__ void join_r(const SweepArgs& a, int g, int64_t row0)
{
    const int64_t i = row0 + threadIdx.x;
    if (threadIdx.x >= kSweepPad) return;
    float sum = 0.f;
    if (i < a.n)
#pragma unroll 4
        for (int z = 0; z < a.splits; ++z) sum += __ldcg(a.part + ((int64_t)z * a.G + g) * a.np + i);
    a.nr[g * a.np + i] = -sum;
}

// (Not inlined: the passes' loops come out slower next to it, MEAN 69 thousand clocks instead of 64.)
template <int MODE>
__device__ __noinline__ void join(const SweepArgs& a, int g, int64_t row0)
{
    if (MODE == SWEEP_LSE) join_lse(a, g, row0);
    else if (MODE == SWEEP_MEAN) join_mean(a, g, row0);
    else join_r(a, g, row0);
}

// Where a row's inputs come from, and its A operand: two bf16 per TMEM column, zeros for a row that is none.
template <int DIN>
__device__ __forceinline__ void load_inputs(uint32_t taddr, const uint16_t* row, bool in)
{
    const uint4* src = reinterpret_cast<const uint4*>(row);
#pragma unroll
    for (int h = 0; h < DIN / 32; ++h) {
        uint32_t v[16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint4 w = in ? ld(src + 4 * h + q) : make_uint4(0, 0, 0, 0);
            v[4 * q] = w.x;
            v[4 * q + 1] = w.y;
            v[4 * q + 2] = w.z;
            v[4 * q + 3] = w.w;
        }
        st16(taddr + 16 * h, v);
    }
    wait_st();
}

// ---- LSE, MEAN, R: the passes
template <int DIN>
struct Sweep {
    static constexpr int AN = DIN == 128 ? 96 : 64;    // columns of an accumulator
    static constexpr int ACCS = DIN == 128 ? 1 : 2;    // accumulators of a block
    static constexpr int TN = ACCS * AN;               // rows of a tile
    static constexpr int ROWB = DIN >= 64 ? 128 : 64;
    static constexpr int BOXES = DIN == 128 ? 2 : 1;
    static constexpr int BOX = TN * ROWB, TILE = BOXES * BOX;
    static constexpr int OFF_STEP = kStages * TILE, STEP = TN * 32, OFF_NUM = OFF_STEP + kStages * STEP, NUM = TN * 4,
                         OFF_ONES = OFF_NUM + kStages * NUM, OFF_BAR = OFF_ONES + AN * 32;
    enum { FULL = 0, EMPTY = kStages, AFULL = 2 * kStages, AFREE = AFULL + kBlocks * ACCS, DRAIN = AFREE + kBlocks * ACCS, COUNT };
    static constexpr int OFF_ABORT = OFF_BAR + COUNT * 8, SMEM = OFF_ABORT + 16;
    static_assert(SMEM <= 226 * 1024 && BOX % 1024 == 0 && OFF_ONES % 16 == 0 && OFF_BAR % 8 == 0, "shared memory");
    static constexpr uint32_t COL_A = kBlocks * TN, COL_ONES = COL_A + kBlocks * (DIN / 2), COL_OWN = COL_ONES + 8;  // (8 of each block)
    static_assert(COL_OWN + 8 * kBlocks <= 512, "TMEM columns");
    static_assert(kSweepPad % TN == 0, "numbers are copied a tile at a time");
};

template <int DIN, int MODE>
__global__ void __launch_bounds__(kSweepThreads, 1) sweep_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ SweepArgs a)
{
    using L = Sweep<DIN>;
    constexpr int TN = L::TN, AN = L::AN, ACCS = L::ACCS;
    constexpr bool kEntriesStand = MODE == SWEEP_MEAN;
    constexpr uint32_t kTileBytes = L::TILE + L::STEP + (MODE == SWEEP_R ? L::NUM : 0);
    extern __shared__ __align__(1024) unsigned char sm[];
    __shared__ uint32_t tmem_slot;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const uint32_t sb = smem_u32(sm);
    auto bar = [&](int i) { return sb + L::OFF_BAR + 8u * (uint32_t)i; };
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + L::OFF_ABORT);
    const int grp = blockIdx.y, split = (int)(blockIdx.x % (uint32_t)a.splits);
    const int64_t n_stand = kEntriesStand ? a.m : a.n, n_stream = kEntriesStand ? a.n : a.m;
    const int64_t row0 = (int64_t)(blockIdx.x / (uint32_t)a.splits) * kRows;
    const int n_blocks = (int)min((n_stand - row0 + 127) / 128, (int64_t)kBlocks);
    const int all_tiles = (int)((n_stream + TN - 1) / TN);
    const int tile0 = (int)((int64_t)all_tiles * split / a.splits), n_tiles = (int)((int64_t)all_tiles * (split + 1) / a.splits) - tile0;

    const int e = warp >> 2;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const int64_t row = row0 + 128 * e + (warp & 3) * 32 + lane;
    const bool in = warp < kReadWarps && row < n_stand;
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            bar_init(bar(L::FULL + s), 1);
            bar_init(bar(L::EMPTY + s), (MODE == SWEEP_R ? 5 : 1) * (uint32_t)n_blocks);  // the products, and who reads h
        }
        for (int i = 0; i < kBlocks * ACCS; ++i) {
            bar_init(bar(L::AFULL + i), 1);
            bar_init(bar(L::AFREE + i), 4);
        }
        bar_init(bar(L::DRAIN), kBlocks);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (MODE != SWEEP_LSE) put_ones(sm + L::OFF_ONES, AN);
    if (warp == kIssueWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    grid_dependency_wait();
    const uint32_t tmem = tmem_slot;
    if (warp < 4 * n_blocks) {
        if (e == 0) store_ones(tmem + lane_base + L::COL_ONES);
        if (MODE != SWEEP_LSE) store_parts(tmem + lane_base + L::COL_OWN + 8 * e, !in ? 0.f : kEntriesStand ? a.b[grp * a.mp + row] : a.nl[grp * a.np + row]);
        load_inputs<DIN>(tmem + lane_base + L::COL_A + e * (DIN / 2), (kEntriesStand ? a.W + ((int64_t)grp * a.m + row) * DIN : a.x + row * DIN), in);
    }
    if (warp < kLoadWarp) {  // (the loading warp is on its way)
        tc_before();
        asm volatile("bar.sync 1, %0;" ::"n"(kLoadWarp * 32) : "memory");
        tc_after();
    }

    LongSum sum;
    float top = -CUDART_INF_F;
    if (warp < kReadWarps) {
        // ------------------------------------------------------------ thread = standing row
        float c = 0.f;  // LSE: log2 of a weight is  s log2(e) + c
        const uint32_t tacc = tmem + lane_base + (uint32_t)(TN * e);
        auto look = [&](uint32_t (&x)[32], const float4* num) {
            F2 u[16];
            if (MODE == SWEEP_LSE) {
                float m0 = __uint_as_float(x[0]), m1 = __uint_as_float(x[1]);
#pragma unroll
                for (int q = 2; q < 30; q += 4) {
                    m0 = max3f(m0, __uint_as_float(x[q]), __uint_as_float(x[q + 1]));
                    m1 = max3f(m1, __uint_as_float(x[q + 2]), __uint_as_float(x[q + 3]));
                }
                m0 = max3f(fmaxf(m0, m1), __uint_as_float(x[30]), __uint_as_float(x[31]));
                if (m0 > top) {
                    const float f = ex2((top - m0) * kLog2e);
                    sum.s *= f;
                    sum.lost *= f;
                    top = m0;
                    c = -m0 * kLog2e;
                }
            }
#pragma unroll
            for (int q = 0; q < 16; ++q) u[q] = MODE == SWEEP_LSE ? fma2(pair(x, 2 * q), both(kLog2e), both(c)) : mul2(pair(x, 2 * q), both(kLog2e));
            F2 part{0.f, 0.f};
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                F2 w{};
                if (MODE == SWEEP_R) {
                    const float4 k = num[q / 2];
                    w = q % 2 ? F2{k.z, k.w} : F2{k.x, k.y};
                }
                if (on_fma(q, MODE == SWEEP_R ? kFmaR : MODE == SWEEP_LSE ? kFmaLse : kFmaMean)) {
                    const Exp2<MODE == SWEEP_R ? 4 : 5> p(u[q]);
                    part = MODE == SWEEP_R ? fma2(mul2(p.p, p.scale), w, part) : fma2(p.p, p.scale, part);
                } else {
                    const F2 p{ex2(u[q].x), ex2(u[q].y)};
                    part = MODE == SWEEP_R ? fma2(p, w, part) : add2(part, p);
                }
            }
            sum.add(part.x + part.y);
        };
        int s = 0;
        for (int t = 0; e < n_blocks && t < n_tiles; ++t) {
            bool ok = true;
            if (MODE == SWEEP_R) ok = bar_wait(bar(L::FULL + s), (t / kStages) & 1, abort_flag);  // (h is to be seen; the products wait themselves)
            const float* num = reinterpret_cast<const float*>(sm + L::OFF_NUM + s * L::NUM);
#pragma unroll
            for (int h = 0; h < ACCS; ++h) {
                const int acc = ACCS * e + h;
                ok = ok && bar_wait(bar(L::AFULL + acc), t & 1, abort_flag);
                if (!ok) break;
                tc_after();
                uint32_t v[AN / 32][32];
#pragma unroll
                for (int c = 0; c < AN / 32; ++c) ld32(tacc + AN * h + 32 * c, v[c]);
#pragma unroll
                for (int c = 0; c < AN / 32; ++c) wait_ld32(v[c]);
                tc_before();
                __syncwarp();
                if (lane == 0) bar_arrive(bar(L::AFREE + acc));
#pragma unroll
                for (int c = 0; c < AN / 32; ++c) look(v[c], reinterpret_cast<const float4*>(num + AN * h + 32 * c));
            }
            if (!ok) break;
            if (MODE == SWEEP_R) {
                __syncwarp();
                if (lane == 0) bar_arrive(bar(L::EMPTY + s));
                if (++s == kStages) s = 0;
            }
        }
        if (MODE == SWEEP_LSE && top > -CUDART_INF_F) sum.s = fabsf(top) < kCoarse ? sum.s * ex2(-fmaf(top, kLog2e, c)) : 1.f;
    } else if (warp < kIssueWarp + kBlocks) {
        // ------------------------------------------------------------ products, one warp per block
        constexpr uint32_t idesc = idesc_bf16(128, AN, false);
        const int blk = warp - kIssueWarp;
        const uint32_t d = tmem + (uint32_t)(TN * blk), at = tmem + L::COL_A + blk * (DIN / 2);
        int s = 0;
        uint32_t par = 0;
        bool ok = true;
        for (int t = 0; ok && blk < n_blocks && t < n_tiles; ++t) {
            ok = bar_wait(bar(L::FULL + s), par, abort_flag);
#pragma unroll
            for (int h = 0; h < ACCS; ++h) {
                if (t > 0) ok = ok && bar_wait(bar(L::AFREE + ACCS * blk + h), (t - 1) & 1, abort_flag);
                if (ok && elect_one()) {
                    tc_after();
                    const uint64_t w = tile_desc<L::ROWB>(sb + s * L::TILE + AN * h * L::ROWB);
#pragma unroll
                    for (int ks = 0; ks < DIN / 16; ++ks)
                        mma_ts(d + AN * h, at + 8 * ks, w + (uint64_t)(((ks & 3) * 32 + (ks >> 2) * L::BOX) >> 4), idesc, ks > 0);
                    const uint64_t ones = step_desc(sb + L::OFF_ONES), step = step_desc(sb + L::OFF_STEP + s * L::STEP + AN * h * 32);
                    const uint32_t own = tmem + L::COL_OWN + 8 * blk;
                    if (MODE == SWEEP_MEAN) mma_ts(d + AN * h, own, ones, idesc, 1u);  // (the bias first)
                    mma_ts(d + AN * h, tmem + L::COL_ONES, step, idesc, 1u);
                    if (MODE == SWEEP_R) mma_ts(d + AN * h, own, ones, idesc, 1u);
                    tc_commit_to(bar(L::AFULL + ACCS * blk + h));
                    if (h == ACCS - 1) tc_commit_to(bar(L::EMPTY + s));
                }
                __syncwarp();
            }
            if (++s == kStages) {
                s = 0;
                par ^= 1;
            }
        }
        // nothing of this CTA may still run on the tensor core at its end
        if (elect_one()) tc_commit_to(bar(L::DRAIN));
        int never = 0;
        if (!bar_wait(bar(L::DRAIN), 0, &never)) *abort_flag = 1;
        __syncwarp();
    } else {
        // ------------------------------------------------------------ tiles
        int issued = 0;
        bool ok = true;
        for (int t = 0; t < n_tiles; ++t) {
            const int s = t % kStages;
            ok = bar_wait(bar(L::EMPTY + s), ((t / kStages) & 1) ^ 1, abort_flag);
            if (!ok) break;
            if (lane == 0) {
                const int64_t c0 = (int64_t)(tile0 + t) * TN;
                expect_bytes(bar(L::FULL + s), kTileBytes);
#pragma unroll
                for (int i = 0; i < L::BOXES; ++i)
                    load_box(sb + s * L::TILE + i * L::BOX, &map, 64 * i, (int)c0, kEntriesStand ? 0 : grp, bar(L::FULL + s));
                load_bytes(sb + L::OFF_STEP + s * L::STEP, kEntriesStand ? a.nl_step + (grp * a.np + c0) * 16 : a.b_step + (grp * a.mp + c0) * 16, L::STEP, bar(L::FULL + s));
                if (MODE == SWEEP_R) load_bytes(sb + L::OFF_NUM + s * L::NUM, a.h + grp * a.mp + c0, L::NUM, bar(L::FULL + s));
            }
            __syncwarp();
            ++issued;
        }
        if (!ok) {  // the copies in flight land before the CTA ends
            int never = 0;
            for (int k = issued > kStages ? issued - kStages : 0; k < issued; ++k) bar_wait(bar(L::FULL + k % kStages), (k / kStages) & 1, &never);
        }
    }

    tc_before();
    __syncthreads();
    tc_after();
    if (warp == kIssueWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    if (in) {
        const int64_t at = ((int64_t)split * a.G + grp) * (kEntriesStand ? a.mp : a.np) + row;
        const float r = *abort_flag ? CUDART_NAN_F : sum.s;
        if (MODE == SWEEP_LSE) reinterpret_cast<float2*>(a.part)[at] = make_float2(*abort_flag ? CUDART_INF_F : top, r);
        else a.part[at] = r;
    }
    if (!a.join_here || !last_of(a.ticket + (int64_t)grp * (gridDim.x / (uint32_t)a.splits) + blockIdx.x / (uint32_t)a.splits, (unsigned)a.splits)) return;
    join<MODE>(a, grp, row0);
}

// The same in a launch of its own.
template <int MODE>
__global__ void __launch_bounds__(kSweepThreads) join_kernel(const __grid_constant__ SweepArgs a)
{
    grid_dependency_wait();
    join<MODE>(a, (int)blockIdx.y, (int64_t)blockIdx.x * kSweepPad);
}

// ---- DX, DW
template <int DIN>
struct Grad {
    static constexpr int BLOCKS = DIN == 128 ? 1 : 2;
    static constexpr int TN = 64;                      // rows of a tile, columns of a score buffer
    static constexpr int READ_WARPS = 8 * BLOCKS, ISSUE_WARP = READ_WARPS, LOAD_WARP = ISSUE_WARP + BLOCKS, THREADS = (LOAD_WARP + 1) * 32;
    static constexpr int ROWB = DIN >= 64 ? 128 : 64;
    static constexpr int BOXES = DIN == 128 ? 2 : 1;
    static constexpr int BOX = TN * ROWB, TILE = BOXES * BOX, STAGES = 8;
    static constexpr int ON = DIN < 64 ? DIN : 64;     // columns of O that one product covers: a box
    static constexpr int OFF_STEP = STAGES * TILE, STEP = TN * 32, OFF_NUM = OFF_STEP + STAGES * STEP, NUM = TN * 4, OFF_SUM = OFF_NUM + STAGES * NUM,
                         OFF_ONES = OFF_SUM + BLOCKS * 128 * 4, OFF_BAR = OFF_ONES + TN * 32;
    enum { FULL = 0, EMPTY = STAGES, SFULL = 2 * STAGES, OFULL = SFULL + 2 * BLOCKS, COUNT = OFULL + BLOCKS };
    static constexpr int OFF_ABORT = OFF_BAR + COUNT * 8, SMEM = OFF_ABORT + 16;
    static_assert(SMEM <= 226 * 1024 && BOX % 1024 == 0 && OFF_ONES % 16 == 0 && OFF_BAR % 8 == 0, "shared memory");
    static constexpr uint32_t COL_O = 2 * TN, COL_A = COL_O + DIN, COL_BLOCK = COL_A + DIN / 2,  // a block's: two buffers, O, inputs
                              COL_ONES = BLOCKS * COL_BLOCK, COL_OWN = COL_ONES + 8;  // (8 of each block)
    static_assert(COL_OWN + 8 * BLOCKS <= 512, "TMEM columns");
    static_assert(kSweepPad % TN == 0, "numbers are copied a tile at a time");
};

template <int DIN, int MODE>
__device__ __forceinline__ void grad_block(const CUtensorMap& map, const SweepArgs& a, const int splits, const uint32_t block, const int of_group, float* const part)
{
    using L = Grad<DIN>;
    constexpr int TN = L::TN;
    constexpr bool kEntriesStand = MODE == SWEEP_DW;
    extern __shared__ __align__(1024) unsigned char sm[];
    __shared__ uint32_t tmem_slot;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const uint32_t sb = smem_u32(sm);
    auto bar = [&](int i) { return sb + L::OFF_BAR + 8u * (uint32_t)i; };
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + L::OFF_ABORT);
    const int split = (int)(block % (uint32_t)splits);
    const int64_t n_stand = kEntriesStand ? a.m : a.n, n_stream = kEntriesStand ? a.n : a.m;
    const int64_t row0 = (int64_t)(block / (uint32_t)splits) * (128 * L::BLOCKS);
    const int n_blocks = (int)min((n_stand - row0 + 127) / 128, (int64_t)L::BLOCKS);
    // tiles of one group after the other (DW: the block's group alone)
    const int per_group = (int)((n_stream + TN - 1) / TN);
    const int64_t all_tiles = (int64_t)per_group * (kEntriesStand ? 1 : a.G);
    const int64_t tile0 = all_tiles * split / splits;
    const int n_tiles = (int)(all_tiles * (split + 1) / splits - tile0);
    const int first_group = kEntriesStand ? of_group : (int)(tile0 / max(per_group, 1)), first_tile = (int)(tile0 - (kEntriesStand ? 0 : (int64_t)first_group * per_group));

    const int e = warp >> 3, buf = (warp >> 2) & 1;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const int at_row = 128 * e + (warp & 3) * 32 + lane;
    const int64_t row = row0 + at_row;
    const bool in = warp < L::READ_WARPS && row < n_stand;
    if (tid == 0) {
        for (int s = 0; s < L::STAGES; ++s) {
            bar_init(bar(L::FULL + s), 1);
            bar_init(bar(L::EMPTY + s), (uint32_t)n_blocks);
        }
        for (int i = 0; i < 2 * L::BLOCKS; ++i) bar_init(bar(L::SFULL + i), 1);
        for (int i = 0; i < L::BLOCKS; ++i) bar_init(bar(L::OFULL + i), 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (kEntriesStand) put_ones(sm + L::OFF_ONES, TN);
    if (warp == L::ISSUE_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    grid_dependency_wait();
    const uint32_t tmem = tmem_slot, tblock = tmem + (uint32_t)e * L::COL_BLOCK;
    if (warp < 4) store_ones(tmem + lane_base + L::COL_ONES);
    if (warp < 8 * n_blocks && buf == 0) {
        if (kEntriesStand) store_parts(tmem + lane_base + L::COL_OWN + 8 * e, in ? a.b[of_group * a.mp + row] : 0.f);
        load_inputs<DIN>(tblock + lane_base + L::COL_A, (kEntriesStand ? a.W + ((int64_t)of_group * a.m + row) * DIN : a.x + row * DIN), in);
    }
    if (warp < L::LOAD_WARP) {  // (the loading warp is on its way)
        tc_before();
        asm volatile("bar.sync 1, %0;" ::"n"(L::LOAD_WARP * 32) : "memory");
        tc_after();
    }

    LongSum sum;
    if (warp < L::READ_WARPS) {
        // ------------------------------------------------------------ weights, thread = standing row, every second tile
        int g = first_group, in_group = first_tile;
        // log2 of a weight is  (s + by) log2(e) + log_own, of which one is zero
        float by = 0.f, log_own = 0.f, h_own = 0.f;
        bool far = false;
        auto take_own = [&] {
            h_own = !in ? 0.f : kEntriesStand ? a.h[g * a.mp + row] : a.nr[g * a.np + row];
            by = !in ? -CUDART_INF_F : kEntriesStand ? 0.f : a.nl[g * a.np + row];
            far = is_far(by);
            log_own = far ? 0.f : by * kLog2e;
        };
        if (n_tiles > 0) take_own();
        const uint32_t ts = tblock + lane_base + (uint32_t)(TN * buf);
        if (buf == 1) ++in_group;
        bool ok = true;
        for (int t = buf; e < n_blocks && t < n_tiles; t += 2, in_group += 2) {
            if (!kEntriesStand && in_group >= per_group) {
                do {
                    in_group -= per_group;
                    ++g;
                } while (in_group >= per_group);
                take_own();
            }
            const int s = t % L::STAGES;
            ok = ok && bar_wait(bar(L::SFULL + 2 * e + buf), (t >> 1) & 1, abort_flag);
            ok = ok && bar_wait(bar(L::FULL + s), (t / L::STAGES) & 1, abort_flag);  // (long complete: the numbers are to be seen)
            if (!ok) {
                weights_sync(2 * e + buf, t);
                continue;
            }
            tc_after();
            const float* num = reinterpret_cast<const float*>(sm + L::OFF_NUM + s * L::NUM);
#pragma unroll
            for (int c = 0; c < TN / 32; ++c) {
                uint32_t v[32], w[16];
                ld32(ts + 32 * c, v);
                wait_ld32(v);
                if (!kEntriesStand && far) move(v, by);
                const float4* n1 = reinterpret_cast<const float4*>(num + 32 * c);
                F2 part{0.f, 0.f};
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float4 hk = n1[q];
                    const F2 u0 = fma2(pair(v, 4 * q), both(kLog2e), both(log_own)), u1 = fma2(pair(v, 4 * q + 2), both(kLog2e), both(log_own));
                    // h_j - r_i, of which one is the thread's own and the other one the column's
                    const F2 d0 = add2({hk.x, hk.y}, both(h_own)), d1 = add2({hk.z, hk.w}, both(h_own));
                    const F2 w0 = mul2(weight<kEntriesStand>(u0, on_fma(2 * q, kFmaGrad)), d0);
                    const F2 w1 = mul2(weight<kEntriesStand>(u1, on_fma(2 * q + 1, kFmaGrad)), d1);
                    if (kEntriesStand) part = add2(part, add2(w0, w1));
                    w[2 * q] = pack_bf16(w0.x, w0.y);
                    w[2 * q + 1] = pack_bf16(w1.x, w1.y);
                }
                if (kEntriesStand) sum.add(part.x + part.y);
                st16(ts + 16 * c, w);  // over columns whose scores have been read
            }
            wait_st();
            tc_before();
            weights_arrive(2 * e + buf, t);
        }
    } else if (warp < L::LOAD_WARP) {
        // ------------------------------------------------------------ products, one warp per block
        // The weighted sum of tile t, then the scores of tile t + 2 into the buffer that it has read: one thread's products run in order.
        constexpr uint32_t idesc_s = idesc_bf16(128, TN, false), idesc_o = idesc_bf16(128, L::ON, true);
        const int blk = warp - L::ISSUE_WARP;
        const uint32_t tb = tmem + (uint32_t)blk * L::COL_BLOCK;
        bool ok = true;
        for (int t = -2; blk < n_blocks && t < n_tiles; ++t) {
            const int nxt = t + 2;
            if (t >= 0) {
                weights_sync(2 * blk + (t & 1), t);
                if (ok && elect_one()) {
                    tc_after();
                    const uint32_t tile = sb + (t % L::STAGES) * L::TILE, tw = tb + (uint32_t)(TN * (t & 1));
#pragma unroll
                    for (int ks = 0; ks < TN / 16; ++ks)
#pragma unroll
                        for (int o = 0; o < L::BOXES; ++o)
                            mma_ts(tb + L::COL_O + 64 * o, tw + 8 * ks, tile_desc<L::ROWB>(tile + o * L::BOX + ks * 16 * L::ROWB), idesc_o, (t > 0) | (ks > 0));
                    tc_commit_to(bar(L::EMPTY + t % L::STAGES));
                }
                __syncwarp();
            }
            if (nxt >= n_tiles) continue;
            ok = ok && bar_wait(bar(L::FULL + nxt % L::STAGES), (nxt / L::STAGES) & 1, abort_flag);
            if (ok && elect_one()) {
                tc_after();
                const uint64_t w = tile_desc<L::ROWB>(sb + (nxt % L::STAGES) * L::TILE);
#pragma unroll
                for (int ks = 0; ks < DIN / 16; ++ks)
                    mma_ts(tb + (uint32_t)(TN * (nxt & 1)), tb + L::COL_A + 8 * ks, w + (uint64_t)(((ks & 3) * 32 + (ks >> 2) * L::BOX) >> 4), idesc_s, ks > 0);
                if (kEntriesStand) mma_ts(tb + (uint32_t)(TN * (nxt & 1)), tmem + L::COL_OWN + 8 * blk, step_desc(sb + L::OFF_ONES), idesc_s, 1u);
                mma_ts(tb + (uint32_t)(TN * (nxt & 1)), tmem + L::COL_ONES, step_desc(sb + L::OFF_STEP + (nxt % L::STAGES) * L::STEP), idesc_s, 1u);
                tc_commit_to(bar(L::SFULL + 2 * blk + (nxt & 1)));
            }
            __syncwarp();
        }
        // O is complete, and nothing of this CTA may still run on the tensor core at its end
        if (elect_one()) tc_commit_to(bar(L::OFULL + blk));
        int never = 0;
        if (!bar_wait(bar(L::OFULL + blk), 0, &never)) *abort_flag = 1;
        __syncwarp();
    } else {
        // ------------------------------------------------------------ tiles
        int issued = 0, g = first_group, in_group = first_tile;
        bool ok = true;
        for (int t = 0; t < n_tiles; ++t, ++in_group) {
            if (!kEntriesStand && in_group == per_group) {
                in_group = 0;
                ++g;
            }
            const int s = t % L::STAGES;
            ok = bar_wait(bar(L::EMPTY + s), ((t / L::STAGES) & 1) ^ 1, abort_flag);
            if (!ok) break;
            if (lane == 0) {
                const int64_t c0 = (int64_t)in_group * TN;
                expect_bytes(bar(L::FULL + s), L::TILE + L::STEP + L::NUM);
#pragma unroll
                for (int i = 0; i < L::BOXES; ++i)
                    load_box(sb + s * L::TILE + i * L::BOX, &map, 64 * i, (int)c0, kEntriesStand ? 0 : g, bar(L::FULL + s));
                load_bytes(sb + L::OFF_STEP + s * L::STEP, kEntriesStand ? a.nl_step + (g * a.np + c0) * 16 : a.b_step + (g * a.mp + c0) * 16, L::STEP, bar(L::FULL + s));
                load_bytes(sb + L::OFF_NUM + s * L::NUM, kEntriesStand ? a.nr + g * a.np + c0 : a.h + g * a.mp + c0, L::NUM, bar(L::FULL + s));
            }
            __syncwarp();
            ++issued;
        }
        if (!ok) {  // the copies in flight land before the CTA ends
            int never = 0;
            for (int k = issued > L::STAGES ? issued - L::STAGES : 0; k < issued; ++k) bar_wait(bar(L::FULL + k % L::STAGES), (k / L::STAGES) & 1, &never);
        }
    }

    float* const half = reinterpret_cast<float*>(sm + L::OFF_SUM);
    if (warp < L::READ_WARPS && buf == 1) half[at_row] = sum.s;
    tc_before();
    __syncthreads();
    tc_after();
    if (warp < 8 * n_blocks && buf == 0) {
        const bool bad = *abort_flag != 0;
        float* out = kEntriesStand ? part + (((int64_t)split * a.G + of_group) * a.m + row) * DIN : part + ((int64_t)split * a.n + row) * DIN;
#pragma unroll
        for (int c = 0; c < DIN / 32; ++c) {
            uint32_t v[32];
            ld32(tblock + lane_base + L::COL_O + 32 * c, v);
            wait_ld32(v);
            if (!in) continue;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                float4 o = make_float4(__uint_as_float(v[4 * q]), __uint_as_float(v[4 * q + 1]), __uint_as_float(v[4 * q + 2]), __uint_as_float(v[4 * q + 3]));
                if (n_tiles == 0) o = make_float4(0.f, 0.f, 0.f, 0.f);
                if (bad) o.x = o.y = o.z = o.w = CUDART_NAN_F;
                reinterpret_cast<float4*>(out)[8 * c + q] = o;
            }
        }
        if (kEntriesStand && in) a.part2[((int64_t)split * a.G + of_group) * a.mp + row] = bad ? CUDART_NAN_F : sum.s + half[at_row];
    }
    tc_before();
    __syncthreads();
    tc_after();
    if (warp == L::ISSUE_WARP)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// The blocks of DX, then those of DW, which want nothing of one another.
template <int DIN>
__global__ void __launch_bounds__(Grad<DIN>::THREADS, 1)
    grad_kernel(const __grid_constant__ CUtensorMap map_W, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ SweepArgs a, const int dx_blocks, const int dw_blocks)
{
    const uint32_t b = blockIdx.x;
    if (b < (uint32_t)dx_blocks) grad_block<DIN, SWEEP_DX>(map_W, a, a.splits, b, 0, a.part);
    else grad_block<DIN, SWEEP_DW>(map_x, a, a.splits_dw, (b - dx_blocks) % (uint32_t)dw_blocks, (int)((b - dx_blocks) / (uint32_t)dw_blocks), a.part_dw);
}

struct Shape {
    int rows, tile;     // standing rows of a CTA, streaming rows of a tile
    double start, join; // what a CTA costs besides its tiles, and what a further split costs, in tiles
};
Shape shape_of(int d, int mode)
{
    if (mode == SWEEP_DX || mode == SWEEP_DW) return Shape{d == 128 ? 128 : 256, 64, 8, 0.5};
    return Shape{kRows, d == 128 ? 96 : 128, 4, 0.25};
}

bool entries_stand(int mode) { return mode == SWEEP_MEAN || mode == SWEEP_DW; }
// Blocks of standing rows, of all groups.
int64_t blocks_of(int64_t n, int G, int d, int64_t m, int mode)
{
    const int rows = shape_of(d, mode).rows;
    return ((entries_stand(mode) ? m : n) + rows - 1) / rows * (mode == SWEEP_DX ? 1 : G);
}
bool map_of(CUtensorMap* map, const void* rows, int64_t n, int G, int d, int tile)
{
    return encode_groups(map, rows, d, n, G, d < 64 ? d : 64, tile, d < 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_128B);
}

template <int DIN>
cudaError_t launch_sweep_t(int mode, const SweepArgs& a, const CUtensorMap& map, dim3 grid, cudaStream_t s)
{
    return launch_granted(s, mode == SWEEP_LSE ? sweep_kernel<DIN, SWEEP_LSE> : mode == SWEEP_MEAN ? sweep_kernel<DIN, SWEEP_MEAN> : sweep_kernel<DIN, SWEEP_R>, grid,
                          kSweepThreads, Sweep<DIN>::SMEM, map, a);
}
template <int DIN>
cudaError_t launch_grad_t(const SweepArgs& a, const CUtensorMap& map_W, const CUtensorMap& map_x, int64_t dx, int64_t dw, cudaStream_t s)
{
    return launch_granted(s, grad_kernel<DIN>, dim3((unsigned)(dx + dw * a.G)), Grad<DIN>::THREADS, Grad<DIN>::SMEM, map_W, map_x, a, (int)dx, (int)dw);
}

}  // namespace

// Blocks that share a standing row's streaming ones: the number with the shortest run, counting whole rounds of blocks over the SMs.
int sweep_splits(int64_t n, int G, int d, int64_t m, int mode)
{
    const Shape sh = shape_of(d, mode);
    const int64_t blocks = blocks_of(n, G, d, m, mode);
    const int64_t tiles = ((entries_stand(mode) ? n : m) + sh.tile - 1) / sh.tile * (mode == SWEEP_DX ? G : 1);
    int best = 1;
    double best_cost = 1e300;
    const int most = (int)std::min<int64_t>(kSweepMaxSplits, std::max<int64_t>(tiles, 1));
    const uint32_t n_tiles = (uint32_t)std::min<int64_t>(tiles, 1 << 30);
    for (int sp = 1; sp <= most; ++sp) {
        const int64_t rounds = (blocks * sp + 147) / 148;
        const double cost = (double)rounds * ((n_tiles + sp - 1) / (uint32_t)sp + sh.start) + sh.join * sp;
        if (cost < best_cost) {
            best_cost = cost;
            best = sp;
        }
    }
    return best;
}

int64_t sweep_tickets(int64_t n, int G, int d, int64_t m, int mode) { return blocks_of(n, G, d, m, mode) + (mode == SWEEP_MEAN ? G : 0); }

cudaError_t launch_sweep(int mode, int d, SweepArgs& a, cudaStream_t s)
{
    const bool entries = entries_stand(mode);
    const int64_t blocks = blocks_of(a.n, a.G, d, a.m, mode);
    if (blocks == 0) return cudaSuccess;
    a.join_here = blocks * a.splits <= 148;
    CUtensorMap map;
    const bool x_streams = entries && a.n > 0;  // (without positions nothing streams, and the map is not used)
    if (!map_of(&map, x_streams ? a.x : a.W, x_streams ? a.n : a.m, x_streams ? 1 : a.G, d, shape_of(d, mode).tile)) return cudaErrorInvalidValue;
    const dim3 grid((unsigned)(blocks / a.G * a.splits), (unsigned)a.G);
    cudaError_t e = d == 32 ? launch_sweep_t<32>(mode, a, map, grid, s) : d == 64 ? launch_sweep_t<64>(mode, a, map, grid, s) : launch_sweep_t<128>(mode, a, map, grid, s);
    if (e != cudaSuccess || a.join_here) return e;
    return launch_kernel(Launch{s, nullptr, nullptr, true}, mode == SWEEP_LSE ? join_kernel<SWEEP_LSE> : mode == SWEEP_MEAN ? join_kernel<SWEEP_MEAN> : join_kernel<SWEEP_R>,
                         dim3((unsigned)(blocks / a.G), (unsigned)a.G), kSweepThreads, 0, 1, a);
}

cudaError_t launch_sweep_grad(int d, SweepArgs& a, cudaStream_t s)
{
    const int64_t dx = blocks_of(a.n, a.G, d, a.m, SWEEP_DX) * a.splits, dw = blocks_of(a.n, a.G, d, a.m, SWEEP_DW) / a.G * a.splits_dw;
    CUtensorMap map_W, map_x;
    const int tile = shape_of(d, SWEEP_DX).tile;
    if (!map_of(&map_W, a.W, a.m, a.G, d, tile) || !map_of(&map_x, a.n ? a.x : a.W, a.n ? a.n : a.m, 1, d, tile)) return cudaErrorInvalidValue;
    return d == 32 ? launch_grad_t<32>(a, map_W, map_x, dx, dw, s) : d == 64 ? launch_grad_t<64>(a, map_W, map_x, dx, dw, s) : launch_grad_t<128>(a, map_W, map_x, dx, dw, s);
}

}  // namespace ckv
