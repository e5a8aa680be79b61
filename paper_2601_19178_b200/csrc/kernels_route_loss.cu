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
// and what streams is shared out among `splits` blocks, whose partial results are joined in their order.
#include <cuda_bf16.h>
#include <math_constants.h>

#include <algorithm>

#include "fit.h"
#include "ptx_helpers.cuh"

namespace ckv {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float bf(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

struct Space {
    // by entry, [G][mp]: bias log2(e), -inf behind the last; h
    float *b2, *h;
    // by position, [G][np]: -lse log2(e), -inf for a position that takes no part; r
    float *nl2, *r;
    uint16_t* xs;        // x with zeros for a position that takes part in no group
    float* part;         // partial results of a pass
    float* part2;
    int32_t* rows_part;  // [blocks][G] positions that take part, and their -log sigmoid(score)
    double* peak_part;
    int32_t* live_part;  // [blocks of 256][G] positions of them that have a weight (scores that are not all -inf)
    float *ds, *sum, *wsum;  // gradient: coefficient of the picked entry [n][G], sums over an entry's positions
    void* seg;
    int64_t bytes;
};
constexpr int kPrepRows = 256;

Space layout(void* ws, int64_t n, int G, int d, int64_t m, bool grad)
{
    Carve c(ws);
    Space s{};
    const int64_t np = sweep_padded(n), mp = sweep_padded(m), blocks = (n + kPrepRows - 1) / kPrepRows;
    s.b2 = c.take<float>(G * mp);
    s.nl2 = c.take<float>(G * np);
    s.xs = c.take<uint16_t>(n * d);
    if (!grad) {
        s.rows_part = c.take<int32_t>(blocks * G);
        s.peak_part = c.take<double>(blocks * G);
        s.live_part = c.take<int32_t>((np + 255) / 256 * G);
        s.part = c.take<float>(std::max(2 * sweep_splits(n, G, d, m, SWEEP_LSE) * G * np, sweep_splits(n, G, d, m, SWEEP_MEAN) * G * mp));
    } else {
        s.h = c.take<float>(G * mp);
        s.r = c.take<float>(G * np);
        s.ds = c.take<float>(n * G);
        s.sum = c.take<float>(G * m * d);
        s.wsum = c.take<float>(G * m);
        s.part = c.take<float>(std::max(std::max(sweep_splits(n, G, d, m, SWEEP_R) * G * np, sweep_splits(n, G, d, m, SWEEP_DX) * n * d), sweep_splits(n, G, d, m, SWEEP_DW) * G * m * d));
        s.part2 = c.take<float>(sweep_splits(n, G, d, m, SWEEP_DW) * G * mp);
        s.seg = c.take<char>(segment_workspace(n, G, d));
    }
    s.bytes = c.used;
    return s;
}

// ---- what the passes read
__global__ void __launch_bounds__(256) entries_kernel(const float* __restrict__ bias, const float* __restrict__ mean,
                                                      const int32_t* __restrict__ offset, float w_balance, int64_t m, int64_t mp,
                                                      float* __restrict__ b2, float* __restrict__ h)
{
    const int64_t j = blockIdx.x * (int64_t)256 + threadIdx.x;
    const int g = blockIdx.y;
    if (j >= mp) return;
    b2[g * mp + j] = j < m ? (bias ? bias[g * m + j] * kLog2e : 0.f) : -CUDART_INF_F;
    if (!h) return;
    const float u = j < m ? mean[g * m + j] * (float)m : 0.f;
    const int32_t rows = offset[g * (m + 1) + m];
    // (an entry that no position gives any weight has p = 0 everywhere, and no gradient)
    h[g * mp + j] = u > 0.f ? w_balance / (float)max(rows, 1) * logf(u) : 0.f;
}

// Positions: x for the passes; forward: the picked entry's score and the sums for the peak loss; gradient: -lse and the picked entry's
// coefficient.
__global__ void __launch_bounds__(kPrepRows) positions_kernel(const RouteLossArgs a, const RouteGradArgs b, Space s, bool grad)
{
    const int64_t i = blockIdx.x * (int64_t)kPrepRows + threadIdx.x, np = (a.n + kSweepPad - 1) / kSweepPad * kSweepPad;
    bool any = false;
    for (int g = 0; g < a.G; ++g) {
        const int32_t k = i < a.n ? a.idx[i * a.G + g] : -1;
        const bool real = k >= 0 && k < a.m;
        any |= real;
        if (grad) {
            if (i < np) {
                const float lse = real ? a.lse[i * a.G + g] : -CUDART_INF_F;
                s.nl2[g * np + i] = lse == -CUDART_INF_F ? lse : -lse * kLog2e;
            }
            if (i < a.n) {
                float v = 0.f;
                if (real) {
                    const int32_t rows = b.offset[(int64_t)g * (a.m + 1) + a.m];
                    v = -b.w_peak / (float)max(rows, 1) * sigmoid(-a.score[i * a.G + g]);
                    if (b.d_score) v += b.d_score[i * a.G + g];
                }
                s.ds[i * a.G + g] = v;
            }
        } else {
            float sc = 0.f;
            if (real) {
                const uint16_t *x = (const uint16_t*)a.x + i * a.d, *w = (const uint16_t*)a.W + ((int64_t)g * a.m + k) * a.d;
                for (int c = 0; c < a.d; ++c) sc = fmaf(bf(x[c]), bf(w[c]), sc);
                if (a.bias) sc += a.bias[(int64_t)g * a.m + k];
            }
            if (i < a.n) a.score[i * a.G + g] = sc;
            // -log sigmoid(sc)
            double soft = real ? (double)(fmaxf(-sc, 0.f) + log1pf(expf(-fabsf(sc)))) : 0.0;
            __shared__ double sum[8];
            __shared__ int count[8];
            const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
            for (int d = 16; d > 0; d /= 2) soft += __shfl_xor_sync(0xffffffffu, soft, d);
            const int rows = __popc(__ballot_sync(0xffffffffu, real));
            if (lane == 0) {
                sum[warp] = soft;
                count[warp] = rows;
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                double t = 0;
                int c = 0;
                for (int w = 0; w < 8; ++w) {
                    t += sum[w];
                    c += count[w];
                }
                s.peak_part[(int64_t)blockIdx.x * a.G + g] = t;
                s.rows_part[(int64_t)blockIdx.x * a.G + g] = c;
            }
            __syncthreads();
        }
    }
    if (i < a.n)
        for (int c = 0; c < a.d; ++c) s.xs[i * a.d + c] = any ? ((const uint16_t*)a.x)[i * a.d + c] : (uint16_t)0;
}

// ---- joins
__global__ void __launch_bounds__(256) lse_join_kernel(const RouteLossArgs a, const SweepArgs p, float* __restrict__ nl2,
                                                       int32_t* __restrict__ live_part)
{
    const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
    const int g = blockIdx.y;
    const int32_t k = i < a.n ? a.idx[i * a.G + g] : -1;
    const bool real = k >= 0 && k < a.m;
    float lse = 0.f, neg = -CUDART_INF_F;
    if (real) {
        float top = -CUDART_INF_F, sum = 0.f;
        for (int z = 0; z < p.splits; ++z) top = fmaxf(top, reinterpret_cast<const float2*>(p.part)[((int64_t)z * a.G + g) * p.np + i].x);
        for (int z = 0; z < p.splits; ++z) {
            const float2 v = reinterpret_cast<const float2*>(p.part)[((int64_t)z * a.G + g) * p.np + i];
            if (v.x > -CUDART_INF_F) sum = fmaf(v.y, exp2f(v.x - top), sum);
        }
        const float l2 = top + log2f(sum);
        if (top == -CUDART_INF_F) lse = top;  // every entry's score is -inf: no weight anywhere
        else {
            lse = l2 * kLn2;
            neg = -l2;
        }
    }
    if (i < p.np) nl2[g * p.np + i] = neg;
    if (i < a.n) a.lse[i * a.G + g] = lse;
    const int live = __syncthreads_count(neg != -CUDART_INF_F);
    if (threadIdx.x == 0) live_part[(int64_t)blockIdx.x * a.G + g] = live;
}

__device__ double block_sum(double v)
{
    __shared__ double part[32];
    __syncthreads();
#pragma unroll
    for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    double t = 0;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) t += part[w];
    return t;
}

// One block per group: the mean weights, and both losses.  mean log(mean m) is summed as (u log u - u + 1) / m with u = mean m:
// the weights sum to one, so that nothing is added, and near balance, where u log u and the sum's other terms cancel, each
// term is as small as what it stands for.  (They sum to less by the share of the positions that have no weight.)
__global__ void __launch_bounds__(1024) mean_join_kernel(const RouteLossArgs a, const SweepArgs p, const Space s, int blocks, int live_blocks)
{
    const int g = blockIdx.x;
    double peak = 0, rows_d = 0, live = 0;
    for (int b = threadIdx.x; b < blocks; b += 1024) {
        peak += s.peak_part[(int64_t)b * a.G + g];
        rows_d += s.rows_part[(int64_t)b * a.G + g];
    }
    for (int b = threadIdx.x; b < live_blocks; b += 1024) live += s.live_part[(int64_t)b * a.G + g];
    peak = block_sum(peak);
    rows_d = block_sum(rows_d);
    live = block_sum(live);
    const float inv = rows_d > 0 ? (float)(1.0 / rows_d) : 0.f;
    double balance = 0;
    for (int64_t j = threadIdx.x; j < a.m; j += 1024) {
        float sum = 0.f;
        for (int z = 0; z < p.splits; ++z) sum += p.part[((int64_t)z * a.G + g) * p.mp + j];
        const float mean = sum * inv;
        a.mean[(int64_t)g * a.m + j] = mean;
        const double u = (double)mean * (double)a.m;
        balance += (u > 0 ? u * log(u) : u * 0) - u + 1;
    }
    balance = block_sum(balance);
    if (threadIdx.x == 0) {
        a.loss[2 * g] = rows_d > 0 ? (float)(balance / (double)a.m + (live - rows_d) / rows_d) : 0.f;
        a.loss[2 * g + 1] = rows_d > 0 ? (float)(peak / rows_d) : 0.f;
    }
}

__global__ void __launch_bounds__(256) r_join_kernel(const SweepArgs p, float* __restrict__ r)
{
    const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
    const int g = blockIdx.y;
    if (i >= p.np) return;
    float sum = 0.f;
    if (i < p.n)
        for (int z = 0; z < p.splits; ++z) sum += p.part[((int64_t)z * p.G + g) * p.np + i];
    r[g * p.np + i] = sum;
}

// dx: the partial sums and the picked entries' rows
__global__ void __launch_bounds__(256) dx_join_kernel(const RouteLossArgs a, const RouteGradArgs b, const SweepArgs p, const float* __restrict__ ds)
{
    for (int64_t e = blockIdx.x * (int64_t)256 + threadIdx.x; e < a.n * a.d; e += (int64_t)gridDim.x * 256) {
        const int64_t i = e / a.d;
        const int c = (int)(e - i * a.d);
        float sum = 0.f;
        for (int z = 0; z < p.splits; ++z) sum += p.part[(int64_t)z * a.n * a.d + e];
        for (int g = 0; g < a.G; ++g) {
            const int32_t k = a.idx[i * a.G + g];
            if (k >= 0 && k < a.m) sum = fmaf(ds[i * a.G + g], bf(((const uint16_t*)a.W)[((int64_t)g * a.m + k) * a.d + c]), sum);
        }
        ((__nv_bfloat16*)b.dx)[e] = __float2bfloat16_rn(sum);
    }
}

__global__ void __launch_bounds__(256) dw_join_kernel(const RouteLossArgs a, const RouteGradArgs b, const SweepArgs p, const Space s)
{
    const int64_t total = a.G * a.m * a.d;
    for (int64_t e = blockIdx.x * (int64_t)256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
        float sum = s.sum[e];
        for (int z = 0; z < p.splits; ++z) sum += p.part[z * total + e];
        ((__nv_bfloat16*)b.dW)[e] = __float2bfloat16_rn(sum);
        if (b.dbias && e % a.d == 0) {
            const int64_t row = e / a.d, g = row / a.m;
            float db = s.wsum[row];
            for (int z = 0; z < p.splits; ++z) db += p.part2[((int64_t)z * a.G + g) * p.mp + (row - g * a.m)];
            b.dbias[row] = db;
        }
    }
}

SweepArgs pass_args(const RouteLossArgs& a, const Space& s)
{
    return SweepArgs{a.n, a.m, sweep_padded(a.n), sweep_padded(a.m), a.G, 1, s.xs, (const uint16_t*)a.W, s.b2, s.h, s.nl2, s.r, s.part, s.part2};
}

}  // namespace

int64_t route_loss_workspace(int64_t n, int G, int d, int64_t m) { return layout(nullptr, n, G, d, m, false).bytes; }
int64_t route_grad_workspace(int64_t n, int G, int d, int64_t m) { return layout(nullptr, n, G, d, m, true).bytes; }

#define TRY(call)                            \
    do {                                     \
        const cudaError_t e_ = (call);       \
        if (e_ != cudaSuccess) return e_;    \
    } while (0)

cudaError_t launch_route_loss(const RouteLossArgs& a, void* ws, cudaStream_t st)
{
    const Space s = layout(ws, a.n, a.G, a.d, a.m, false);
    SweepArgs p = pass_args(a, s);
    const Launch l{st, nullptr, nullptr};
    const unsigned blocks = (unsigned)((a.n + kPrepRows - 1) / kPrepRows), G = (unsigned)a.G;
    TRY(launch_kernel(l, entries_kernel, dim3((unsigned)((p.mp + 255) / 256), G), 256, 0, 1, a.bias, nullptr, nullptr, 0.f, a.m, p.mp, s.b2, nullptr));
    if (a.n) TRY(launch_kernel(l, positions_kernel, dim3(blocks), kPrepRows, 0, 1, a, RouteGradArgs{}, s, false));
    TRY(launch_sweep(SWEEP_LSE, a.d, p, st));
    if (a.n) TRY(launch_kernel(l, lse_join_kernel, dim3((unsigned)((p.np + 255) / 256), G), 256, 0, 1, a, p, s.nl2, s.live_part));
    TRY(launch_sweep(SWEEP_MEAN, a.d, p, st));
    return launch_kernel(l, mean_join_kernel, dim3(G), 1024, 0, 1, a, p, s, (int)blocks, (int)((p.np + 255) / 256));
}

cudaError_t launch_route_grad(const RouteLossArgs& a, const RouteGradArgs& b, void* ws, cudaStream_t st)
{
    const Space s = layout(ws, a.n, a.G, a.d, a.m, true);
    SweepArgs p = pass_args(a, s);
    const Launch l{st, nullptr, nullptr};
    const unsigned G = (unsigned)a.G;
    TRY(launch_kernel(l, entries_kernel, dim3((unsigned)((p.mp + 255) / 256), G), 256, 0, 1, a.bias, a.mean, b.offset, b.w_balance, a.m, p.mp, s.b2, s.h));
    if (a.n) TRY(launch_kernel(l, positions_kernel, dim3((unsigned)((p.np + kPrepRows - 1) / kPrepRows)), kPrepRows, 0, 1, a, b, s, true));
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
    TRY(launch_sweep(SWEEP_R, a.d, p, st));
    if (a.n) TRY(launch_kernel(l, r_join_kernel, dim3((unsigned)((p.np + 255) / 256), G), 256, 0, 1, p, s.r));
    TRY(launch_sweep(SWEEP_DX, a.d, p, st));
    if (a.n) TRY(launch_kernel(l, dx_join_kernel, dim3((unsigned)std::min<int64_t>((a.n * a.d + 255) / 256, 148 * 16)), 256, 0, 1, a, b, p, s.ds));
    TRY(launch_sweep(SWEEP_DW, a.d, p, st));
    return launch_kernel(l, dw_join_kernel, dim3((unsigned)std::min<int64_t>((a.G * a.m * a.d + 255) / 256, 148 * 16)), 256, 0, 1, a, b, p, s);
}

}  // namespace ckv
