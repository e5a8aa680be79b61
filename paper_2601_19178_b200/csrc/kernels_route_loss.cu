// Losses of the prefill router (Sec. 4.3) and their gradient.
//
//   M_ij = x_i . W_j + b_j,  lse_i = log sum_j exp M_ij,  p_ij = exp(M_ij - lse_i)      (one router per group)
//   mean_j = (1 / rows) sum_i p_ij,  balance = sum_j mean_j log(mean_j m),  peak = -(1 / rows) sum_i log sigmoid(M_{i, I_i})
//   h_j = w_balance log(mean_j m) / rows,  r_i = sum_j p_ij h_j,  T_ij = p_ij (h_j - r_i)
//   dM_ij = T_ij + [j = I_i] (d_score_i - w_peak sigmoid(-M_{i, I_i}) / rows)
//   dx = sum_g dM W,  dW = dM^T x,  db = sum_i dM
//
// The score matrix never lies in memory: every pass recomputes its tiles.  A pass has one side's rows stand still, one per
// thread, and the other side's stream by:
//   LSE   positions stand, entries stream:  running maximum and sum
//   MEAN  entries stand, positions stream:  sum_i p_ij
//   R     positions stand, entries stream:  sum_j p_ij h_j
//   DX    positions stand, entries of all groups stream:  sum_j T_ij W_j
//   DW    entries stand, positions stream:  sum_i T_ij x_i, sum_i T_ij
// and what streams is shared out among `splits` blocks, whose partial results are joined in the order of those blocks: by the last
// of them, or in a launch of its own (kernels_route_sweep.cu); those of DX and DW together, in grad_join_kernel.
#include <cuda_bf16.h>
#include <math_constants.h>

#include <algorithm>

#include "fit.h"
#include "ptx_helpers.cuh"

namespace ckv {
namespace {

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

struct Space {
    // by entry, [G][mp]: bias, -inf behind the last; h
    float *b, *h;
    // by position, [G][np]: -lse, -inf for a position that takes no part; -r
    float *nl, *nr;
    uint16_t *b_step, *nl_step;  // b and nl as operands of a product
    uint16_t* xs;        // x with zeros for a position that takes part in no group, see prepare_kernel
    float* spoilt;       // forward, by position: NaN where its inputs are not numbers and are zeros in xs, else 0
    float* part;         // partial results of a pass
    float *part_dw, *part2;
    int32_t *rows_part, *live_part;  // forward, see SweepArgs
    double *peak_part, *balance_part;
    float *ds, *sum, *wsum;  // gradient: coefficient of the picked entry [n][G], sums over an entry's positions
    void* seg;
    unsigned* ticket[5];     // of the passes LSE, MEAN and R, back to back
    int64_t n_tickets;
    int splits[5];           // of each pass
    int64_t bytes;
};

Space layout(void* ws, int64_t n, int G, int d, int64_t m, bool grad)
{
    Carve c(ws);
    Space s{};
    const int64_t np = sweep_padded(n), mp = sweep_padded(m);
    for (int mode = grad ? SWEEP_R : SWEEP_LSE; mode <= (grad ? SWEEP_DW : SWEEP_MEAN); ++mode) s.splits[mode] = sweep_splits(n, G, d, m, mode);
    for (int mode = grad ? SWEEP_R : SWEEP_LSE; mode <= (grad ? SWEEP_R : SWEEP_MEAN); ++mode) s.n_tickets += sweep_tickets(n, G, d, m, mode);
    unsigned* ticket = c.take<unsigned>(s.n_tickets);
    for (int mode = grad ? SWEEP_R : SWEEP_LSE; ticket && mode <= (grad ? SWEEP_R : SWEEP_MEAN); ++mode) {
        s.ticket[mode] = ticket;
        ticket += sweep_tickets(n, G, d, m, mode);
    }
    s.b = c.take<float>(G * mp);
    s.nl = c.take<float>(G * np);
    s.b_step = c.take<uint16_t>(G * mp * 16);
    s.nl_step = c.take<uint16_t>(G * np * 16);
    s.xs = c.take<uint16_t>(n * d);
    if (!grad) {
        s.spoilt = c.take<float>(n);
        s.rows_part = c.take<int32_t>(sweep_blocks(n) * G);
        s.live_part = c.take<int32_t>(sweep_blocks(n) * G);
        s.peak_part = c.take<double>(sweep_blocks(n) * G);
        s.balance_part = c.take<double>(sweep_blocks(m) * G);
        s.part = c.take<float>(std::max(2 * (int64_t)s.splits[SWEEP_LSE] * G * np, (int64_t)s.splits[SWEEP_MEAN] * G * mp));
    } else {
        s.h = c.take<float>(G * mp);
        s.nr = c.take<float>(G * np);
        s.ds = c.take<float>(n * G);
        s.sum = c.take<float>(G * m * d);
        s.wsum = c.take<float>(G * m);
        s.part = c.take<float>(std::max((int64_t)s.splits[SWEEP_R] * G * np, (int64_t)s.splits[SWEEP_DX] * n * d));
        s.part_dw = c.take<float>((int64_t)s.splits[SWEEP_DW] * G * m * d);
        s.part2 = c.take<float>((int64_t)s.splits[SWEEP_DW] * G * mp);
        s.seg = c.take<char>(segment_workspace(n, G, d));
    }
    s.bytes = c.used;
    return s;
}

// A bias of this or less takes its entry out, as masks by a type's lowest value want it, also where it is all entries' bias.
constexpr float kTakenOut = -1048576.f;

// ---- what the passes read
__device__ __forceinline__ void prepare_entry(const RouteLossArgs& a, const RouteGradArgs& b, const Space& s, int64_t mp, int g, int64_t j)
{
    if (j >= mp) return;
    float bias = j < a.m ? (a.bias ? a.bias[g * a.m + j] : 0.f) : -CUDART_INF_F;
    if (bias <= kTakenOut) bias = -CUDART_INF_F;
    s.b[g * mp + j] = bias;
    put_step(s.b_step, g * mp + j, bias);
    if (!s.h) return;
    const float u = j < a.m ? a.mean[g * a.m + j] * (float)a.m : 0.f;
    const int32_t rows = b.offset[g * (a.m + 1) + a.m];
    // (an entry that no position gives any weight has p = 0 everywhere, and no gradient)
    s.h[g * mp + j] = u > 0.f ? b.w_balance / (float)max(rows, 1) * logf(u) : 0.f;
}

// Positions: x for the passes (zeros for one that takes part in no group, whose inputs may be anything; also for one that takes part in some groups
// and not in others if its inputs are not finite: they spoil the former by its lse, which is not a number, and not the latter); forward: the picked entry's
// score (rows of W by index, 32768 positions x 4 groups x 128 bytes 22 us: latency); gradient: -lse and the picked entry's coefficient (13 us).  A position to D / 8 lanes, 16 bytes of it to each.  The first
// `entry_blocks` blocks, as many for each group, prepare the entries instead.
template <int D, bool GRAD>
__global__ void __launch_bounds__(256) prepare_kernel(const RouteLossArgs a, const RouteGradArgs b, const Space s, int64_t np, int64_t mp,
                                                      int entry_blocks, bool whole)
{
    constexpr int LANES = D / 8;
    grid_dependency_wait();
    for (int64_t t = blockIdx.x * (int64_t)256 + threadIdx.x; t < s.n_tickets; t += (int64_t)gridDim.x * 256) (GRAD ? s.ticket[SWEEP_R] : s.ticket[SWEEP_LSE])[t] = 0;
    if ((int)blockIdx.x < entry_blocks) {
        const int per_group = entry_blocks / a.G;
        prepare_entry(a, b, s, mp, (int)blockIdx.x / per_group, (int64_t)((int)blockIdx.x % per_group) * 256 + threadIdx.x);
        return;
    }
    const int64_t i = (int64_t)((int)blockIdx.x - entry_blocks) * (256 / LANES) + threadIdx.x / LANES;
    const int sub = threadIdx.x % LANES;
    const bool there = i < a.n;
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (there) {
        const uint16_t* x = (const uint16_t*)a.x + i * D + 8 * sub;
        if (whole) raw = ld(reinterpret_cast<const uint4*>(x));
        else {
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = x[2 * q] | (uint32_t)x[2 * q + 1] << 16;
            raw = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    const uint32_t xw[4] = {raw.x, raw.y, raw.z, raw.w};
    // what all lanes of the position have found: bit 0, it takes part in a group; 1, not in another one; 2, inputs that are not finite
    int found = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) found |= (xw[q] & 0x7f80u) == 0x7f80u || (xw[q] & 0x7f800000u) == 0x7f800000u ? 4 : 0;
    auto share = [&] {
#pragma unroll
        for (int d = LANES / 2; d > 0; d /= 2) found |= __shfl_xor_sync(0xffffffffu, found, d);
    };
    if (GRAD) {
        for (int g = sub; g < a.G; g += LANES) {
            const int32_t k = there ? ld(a.idx + i * a.G + g) : -1;
            found |= k >= 0 && k < a.m ? 1 : 2;
        }
        share();
        for (int g = sub; g < a.G; g += LANES) {
            const int32_t k = there ? ld(a.idx + i * a.G + g) : -1;
            const bool real = k >= 0 && k < a.m;
            if (i < np) {
                const float lse = !real ? -CUDART_INF_F : found == 7 ? CUDART_NAN_F : ld(a.lse + i * a.G + g);
                const float nl = lse == -CUDART_INF_F ? lse : -lse;
                s.nl[g * np + i] = nl;
                put_step(s.nl_step, g * np + i, nl);
            }
            if (there) {
                float v = 0.f;
                if (real) {
                    const int32_t rows = ld(b.offset + (int64_t)g * (a.m + 1) + a.m);
                    v = -b.w_peak / (float)max(rows, 1) * sigmoid(-ld(a.score + i * a.G + g));
                    if (b.d_score) v += ld(b.d_score + i * a.G + g);
                }
                s.ds[i * a.G + g] = v;
            }
        }
    } else {
#pragma unroll 2
        for (int g = 0; g < a.G; ++g) {
            const int32_t k = there ? ld(a.idx + i * a.G + g) : -1;
            const bool real = k >= 0 && k < a.m;
            found |= real ? 1 : 2;
            float sc = 0.f;
            if (real) {
                const uint4 w = ld(reinterpret_cast<const uint4*>((const uint16_t*)a.W + ((int64_t)g * a.m + k) * D) + sub);
                const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    sc = fmaf(__uint_as_float(xw[q] << 16), __uint_as_float(ww[q] << 16), sc);
                    sc = fmaf(__uint_as_float(xw[q] & 0xffff0000u), __uint_as_float(ww[q] & 0xffff0000u), sc);
                }
            }
#pragma unroll
            for (int d = LANES / 2; d > 0; d /= 2) sc += __shfl_xor_sync(0xffffffffu, sc, d);
            if (sub == 0 && there) a.score[i * a.G + g] = real && a.bias ? sc + ld(a.bias + (int64_t)g * a.m + k) : sc;
        }
        share();
        if (sub == 0 && there) s.spoilt[i] = found == 7 ? CUDART_NAN_F : 0.f;
    }
    if (there) reinterpret_cast<uint4*>(s.xs + i * D)[sub] = (found & 1) && found != 7 ? raw : make_uint4(0, 0, 0, 0);
}

// ---- joins
// Eight elements of a row: partial sums added in their order, and rounded.
__device__ __forceinline__ void add8(float (&v)[8], const float* p)
{
    const float4 x = ld(reinterpret_cast<const float4*>(p)), y = ld(reinterpret_cast<const float4*>(p) + 1);
    v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w, v[4] += y.x, v[5] += y.y, v[6] += y.z, v[7] += y.w;
}
__device__ __forceinline__ void put8(uint16_t* out, const float (&v)[8], bool whole)
{
    const uint4 w = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    if (whole) *reinterpret_cast<uint4*>(out) = w;
    else {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int q = 0; q < 8; ++q) out[q] = (uint16_t)(u[q / 2] >> (16 * (q & 1)));
    }
}

// Bound by memory, which gives the partial sums back: 200 positions x 1024 entries x 2 groups 4.7 us, 10007 x 4099 x 3 at d_in = 128 10 us.
// The first dx_blocks blocks: dx, the partial sums and the picked entries' rows.  The others: dW and db, the partial sums and the sums over the
// positions that picked the entry.
__global__ void __launch_bounds__(256) grad_join_kernel(const RouteLossArgs a, const RouteGradArgs b, const SweepArgs p, int dx_blocks)
{
    grid_dependency_wait();
    float v[8] = {};
    if ((int)blockIdx.x < dx_blocks) {
        const int64_t e = (blockIdx.x * (int64_t)256 + threadIdx.x) * 8, total = a.n * a.d;
        if (e >= total) return;
        const int64_t i = e / a.d;
        const int c = (int)(e - i * a.d);
#pragma unroll 4
        for (int z = 0; z < p.splits; ++z) add8(v, p.part + z * total + e);
#pragma unroll 4
        for (int g = 0; g < a.G; ++g) {
            const int32_t k = ld(a.idx + i * a.G + g);
            if (k < 0 || k >= a.m) continue;
            const float f = ld(p.ds + i * a.G + g);
            const uint4 w = ld(reinterpret_cast<const uint4*>(p.W + ((int64_t)g * a.m + k) * a.d + c));
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                v[2 * q] = fmaf(f, __uint_as_float(u[q] << 16), v[2 * q]);
                v[2 * q + 1] = fmaf(f, __uint_as_float(u[q] & 0xffff0000u), v[2 * q + 1]);
            }
        }
        put8((uint16_t*)b.dx + e, v, ((uintptr_t)b.dx & 15) == 0);
        return;
    }
    const int64_t e = ((int64_t)((int)blockIdx.x - dx_blocks) * 256 + threadIdx.x) * 8, total = a.G * a.m * a.d;
    if (e >= total) return;
    add8(v, p.sum + e);
#pragma unroll 4
    for (int z = 0; z < p.splits_dw; ++z) add8(v, p.part_dw + z * total + e);
    put8((uint16_t*)b.dW + e, v, ((uintptr_t)b.dW & 15) == 0);
    if (b.dbias && e % a.d == 0) {
        const int64_t row = e / a.d, g = row / a.m;
        float db = ld(p.wsum + row);
        for (int z = 0; z < p.splits_dw; ++z) db += ld(p.part2 + ((int64_t)z * a.G + g) * p.mp + (row - g * a.m));
        b.dbias[row] = db;
    }
}

template <bool GRAD>
cudaError_t launch_prepare(const RouteLossArgs& a, const RouteGradArgs& b, const Space& s, int64_t rows, int64_t np, int64_t mp, cudaStream_t st)
{
    const bool whole = ((uintptr_t)a.x & 15) == 0;
    const int entry_blocks = (int)((mp + 255) / 256) * a.G;
    return launch_kernel(Launch{st, nullptr, nullptr, true},
                         a.d == 32 ? prepare_kernel<32, GRAD> : a.d == 64 ? prepare_kernel<64, GRAD> : prepare_kernel<128, GRAD>,
                         dim3((unsigned)(entry_blocks + (rows * (a.d / 8) + 255) / 256)), 256, 0, 1, a, b, s, np, mp, entry_blocks, whole);
}

SweepArgs pass_args(const RouteLossArgs& a, const Space& s)
{
    SweepArgs p{};
    p.n = a.n, p.m = a.m, p.np = sweep_padded(a.n), p.mp = sweep_padded(a.m);
    p.G = a.G;
    p.x = s.xs, p.W = (const uint16_t*)a.W;
    p.b = s.b, p.h = s.h, p.nl = s.nl, p.nr = s.nr, p.b_step = s.b_step, p.nl_step = s.nl_step;
    p.part = s.part, p.part_dw = s.part_dw, p.part2 = s.part2;
    p.spoilt = s.spoilt;
    p.idx = a.idx, p.score = a.score, p.lse = a.lse, p.mean = a.mean, p.loss = a.loss;
    p.rows_part = s.rows_part, p.live_part = s.live_part, p.peak_part = s.peak_part, p.balance_part = s.balance_part;
    p.ds = s.ds, p.sum = s.sum, p.wsum = s.wsum;
    return p;
}
cudaError_t pass(int mode, int d, SweepArgs& p, const Space& s, cudaStream_t st)
{
    p.ticket = s.ticket[mode];
    p.splits = s.splits[mode];
    return launch_sweep(mode, d, p, st);
}

}  // namespace

int64_t route_loss_workspace(int64_t n, int G, int d, int64_t m) { return layout(nullptr, n, G, d, m, false).bytes; }
int64_t route_grad_workspace(int64_t n, int G, int d, int64_t m) { return layout(nullptr, n, G, d, m, true).bytes; }

#define TRY(call)                            \
    do {                                     \
        const cudaError_t e_ = (call);       \
        if (e_ != cudaSuccess) return e_;    \
    } while (0)

cudaError_t launch_route_loss(const RouteLossArgs& a, void* ws, int64_t bytes, cudaStream_t st)
{
    const Space s = layout(ws, a.n, a.G, a.d, a.m, false);
    if (bytes < s.bytes) return kNoRoom;
    SweepArgs p = pass_args(a, s);
    TRY(launch_prepare<false>(a, RouteGradArgs{}, s, a.n, p.np, p.mp, st));
    TRY(pass(SWEEP_LSE, a.d, p, s, st));
    return pass(SWEEP_MEAN, a.d, p, s, st);
}

cudaError_t launch_route_grad(const RouteLossArgs& a, const RouteGradArgs& b, void* ws, int64_t bytes, cudaStream_t st)
{
    const Space s = layout(ws, a.n, a.G, a.d, a.m, true);
    if (bytes < s.bytes) return kNoRoom;
    SweepArgs p = pass_args(a, s);
    TRY(launch_prepare<true>(a, b, s, a.n ? p.np : 0, p.np, p.mp, st));
    SegmentArgs seg{};
    seg.order = b.order;
    seg.offset = b.offset;
    seg.rows = s.xs;
    seg.stride = a.d;
    seg.n = a.n;
    seg.m = a.m;
    seg.G = a.G;
    seg.width = a.d;
    seg.score = s.ds;
    seg.sum = s.sum;
    seg.weight_sum = s.wsum;
    TRY(launch_segment_sum(CKV_BF16, seg, s.seg, st));
    TRY(pass(SWEEP_R, a.d, p, s, st));
    p.splits = s.splits[SWEEP_DX];
    p.splits_dw = s.splits[SWEEP_DW];
    TRY(launch_sweep_grad(a.d, p, st));
    const int64_t dx_blocks = (a.n * a.d / 8 + 255) / 256, dw_blocks = (a.G * a.m * a.d / 8 + 255) / 256;
    return launch_kernel(Launch{st, nullptr, nullptr, true}, grad_join_kernel, dim3((unsigned)(dx_blocks + dw_blocks)), 256, 0, 1, a, b, p, (int)dx_blocks);
}

}  // namespace ckv
