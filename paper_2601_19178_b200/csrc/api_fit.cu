// Entry points of the training side (include/ckv.h, "Fitting the router and the pool"): argument checks, and the launches.
#include "fit.h"
#include "host_util.h"

using namespace ckv;

namespace {

constexpr int kMaxGroups = 65535;  // a grid dimension

// Sizes every call has.
ckv_status check_sizes(int32_t device, int32_t n, int32_t n_groups, int32_t n_entries)
{
    if (device < 0 || n < 0 || n_groups < 1 || n_entries < 1) return CKV_ERR_INVALID_ARG;
    return n_groups > kMaxGroups ? CKV_ERR_UNSUPPORTED : CKV_OK;
}

struct Arg {
    const void* p;
    int align;
    bool optional = false;
};
// Memory of the call's device (or managed), aligned to its elements.
template <typename... A>
bool on_device(int device, const A&... args)
{
    for (const Arg& a : {args...}) {
        if (!a.p) {
            if (a.optional) continue;
            return false;
        }
        if ((uintptr_t)a.p % (uintptr_t)a.align) return false;
        const int owner = memory_of(a.p);
        if (owner != device && owner != kManagedMemory) return false;
    }
    return true;
}

ckv_status check_workspace(int device, const void* ws, int64_t have, int64_t need)
{
    return have < need || (need > 0 && !on_device(device, Arg{ws, 256})) ? CKV_ERR_INVALID_ARG : CKV_OK;
}

ckv_status status_of(cudaError_t e)
{
    if (e == cudaSuccess) return CKV_OK;
    cudaGetLastError();
    return e == kNoRoom ? CKV_ERR_INVALID_ARG : CKV_ERR_CUDA;
}

bool route_width(int32_t d_in) { return d_in == 32 || d_in == 64 || d_in == 128; }

ckv_status check_gather(int32_t device, int32_t dtype, int32_t n, int32_t n_groups, int32_t head_dim, int32_t d_shared, int32_t n_entries)
{
    const ckv_status st = check_sizes(device, n, n_groups, n_entries);
    if (st != CKV_OK) return st;
    if (dtype != CKV_F32 && dtype != CKV_BF16) return CKV_ERR_INVALID_ARG;
    if (head_dim != 16 && head_dim != 32 && head_dim != 64 && head_dim != 128) return CKV_ERR_UNSUPPORTED;
    if (d_shared < 1 || d_shared > head_dim) return CKV_ERR_SHAPE;
    return (int64_t)n_groups * n_entries >= 0xffffffffll ? CKV_ERR_UNSUPPORTED : CKV_OK;  // pool rows are counted in 32 bits
}

}  // namespace

namespace ckv {

SmemGrants* fit_grants()
{
    constexpr int kDevices = 16;
    static thread_local SmemGrants grants[kDevices];
    int device = -1;
    return cudaGetDevice(&device) == cudaSuccess && device >= 0 && device < kDevices ? &grants[device] : nullptr;
}

}  // namespace ckv

extern "C" {

ckv_status ckv_sort_indices_bytes(int32_t n, int32_t n_groups, int32_t n_entries, int64_t* bytes)
{
    if (!bytes) return CKV_ERR_INVALID_ARG;
    const ckv_status st = check_sizes(0, n, n_groups, n_entries);
    if (st == CKV_OK) *bytes = sort_workspace(n, n_groups, n_entries);
    return st;
}

ckv_status ckv_sort_indices(int32_t device, int32_t n, int32_t n_groups, int32_t n_entries, const int32_t* idx, int32_t* order,
                            int32_t* offset, void* workspace, int64_t workspace_bytes, void* stream)
{
    ckv_status st = check_sizes(device, n, n_groups, n_entries);
    if (st != CKV_OK) return st;
    DeviceGuard dg(device);
    if (!dg.ok) return CKV_ERR_CUDA;
    if (!on_device(device, Arg{idx, 4, n == 0}, Arg{order, 4, n == 0}, Arg{offset, 4})) return CKV_ERR_INVALID_ARG;
    st = check_workspace(device, workspace, workspace_bytes, sort_workspace(n, n_groups, n_entries));
    if (st != CKV_OK) return st;
    return status_of(launch_sort_indices(n, n_groups, n_entries, idx, order, offset, workspace, (cudaStream_t)stream));
}

ckv_status ckv_route_loss_bytes(int32_t n, int32_t n_groups, int32_t d_in, int32_t n_entries, int64_t* forward, int64_t* grad)
{
    if (!forward || !grad) return CKV_ERR_INVALID_ARG;
    const ckv_status st = check_sizes(0, n, n_groups, n_entries);
    if (st != CKV_OK) return st;
    if (!route_width(d_in)) return CKV_ERR_UNSUPPORTED;
    *forward = route_loss_workspace(n, n_groups, d_in, n_entries);
    *grad = route_grad_workspace(n, n_groups, d_in, n_entries);
    return CKV_OK;
}

ckv_status ckv_route_loss(int32_t device, int32_t n, int32_t n_groups, int32_t d_in, int32_t n_entries, const void* x, const void* W,
                          const float* bias, const int32_t* idx, float* loss, float* lse, float* score, float* mean, void* workspace,
                          int64_t workspace_bytes, void* stream)
{
    ckv_status st = check_sizes(device, n, n_groups, n_entries);
    if (st != CKV_OK) return st;
    if (!route_width(d_in)) return CKV_ERR_UNSUPPORTED;
    DeviceGuard dg(device);
    if (!dg.ok) return CKV_ERR_CUDA;
    const bool none = n == 0;
    if (!on_device(device, Arg{x, 2, none}, Arg{W, 16}, Arg{bias, 4, true}, Arg{idx, 4, none}, Arg{loss, 4}, Arg{lse, 4, none},
                   Arg{score, 4, none}, Arg{mean, 4}))
        return CKV_ERR_INVALID_ARG;
    if (!on_device(device, Arg{workspace, 256})) return CKV_ERR_INVALID_ARG;
    const RouteLossArgs a{n, n_entries, n_groups, d_in, x, W, bias, idx, loss, lse, score, mean};
    return status_of(launch_route_loss(a, workspace, workspace_bytes, (cudaStream_t)stream));
}

ckv_status ckv_route_loss_grad(int32_t device, int32_t n, int32_t n_groups, int32_t d_in, int32_t n_entries, const void* x,
                               const void* W, const float* bias, const int32_t* idx, const int32_t* order, const int32_t* offset,
                               const float* lse, const float* score, const float* mean, float balance_weight, float peak_weight,
                               const float* d_score, void* dx, void* dW, float* dbias, void* workspace, int64_t workspace_bytes,
                               void* stream)
{
    ckv_status st = check_sizes(device, n, n_groups, n_entries);
    if (st != CKV_OK) return st;
    if (!route_width(d_in)) return CKV_ERR_UNSUPPORTED;
    DeviceGuard dg(device);
    if (!dg.ok) return CKV_ERR_CUDA;
    const bool none = n == 0;
    if (!on_device(device, Arg{x, 2, none}, Arg{W, 16}, Arg{bias, 4, true}, Arg{idx, 4, none}, Arg{order, 4, none}, Arg{offset, 4},
                   Arg{lse, 4, none}, Arg{score, 4, none}, Arg{mean, 4}, Arg{d_score, 4, true}, Arg{dx, 2, none}, Arg{dW, 2},
                   Arg{dbias, 4, true}))
        return CKV_ERR_INVALID_ARG;
    if (!on_device(device, Arg{workspace, 256})) return CKV_ERR_INVALID_ARG;
    const RouteLossArgs a{n, n_entries, n_groups, d_in, x, W, bias, idx, nullptr, const_cast<float*>(lse), const_cast<float*>(score),
                          const_cast<float*>(mean)};
    const RouteGradArgs b{order, offset, balance_weight, peak_weight, d_score, dx, dW, dbias};
    return status_of(launch_route_grad(a, b, workspace, workspace_bytes, (cudaStream_t)stream));
}

ckv_status ckv_gather_bytes(int32_t dtype, int32_t n, int32_t n_groups, int32_t head_dim, int32_t d_shared, int32_t n_entries,
                            int64_t* bytes)
{
    if (!bytes) return CKV_ERR_INVALID_ARG;
    const ckv_status st = check_gather(0, dtype, n, n_groups, head_dim, d_shared, n_entries);
    if (st == CKV_OK) *bytes = gather_workspace(dtype, n, n_groups, head_dim, d_shared, n_entries);
    return st;
}

ckv_status ckv_gather(int32_t device, int32_t dtype, int32_t n, int32_t n_groups, int32_t head_dim, int32_t d_shared, int32_t n_entries,
                      const void* pool, const int32_t* idx, const void* user, const float* score, void* out, void* workspace,
                      int64_t workspace_bytes, void* stream)
{
    ckv_status st = check_gather(device, dtype, n, n_groups, head_dim, d_shared, n_entries);
    if (st != CKV_OK) return st;
    if (n == 0) return CKV_OK;
    DeviceGuard dg(device);
    if (!dg.ok) return CKV_ERR_CUDA;
    const int e = dtype == CKV_F32 ? 4 : 2;
    if (!on_device(device, Arg{pool, e}, Arg{idx, 4}, Arg{user, e, d_shared == head_dim}, Arg{score, 4, true}, Arg{out, e})) return CKV_ERR_INVALID_ARG;
    st = check_workspace(device, workspace, workspace_bytes, gather_workspace(dtype, n, n_groups, head_dim, d_shared, n_entries));
    if (st != CKV_OK) return st;
    return status_of(launch_gather(dtype, n, n_groups, head_dim, d_shared, n_entries, pool, idx, user, score, out, workspace, (cudaStream_t)stream));
}

ckv_status ckv_gather_grad_bytes(int32_t n, int32_t n_groups, int32_t head_dim, int64_t* bytes)
{
    if (!bytes) return CKV_ERR_INVALID_ARG;
    const ckv_status st = check_gather(0, CKV_F32, n, n_groups, head_dim, 1, 1);
    if (st == CKV_OK) *bytes = segment_workspace(n, n_groups, head_dim);
    return st;
}

ckv_status ckv_gather_grad(int32_t device, int32_t dtype, int32_t n, int32_t n_groups, int32_t head_dim, int32_t d_shared,
                           int32_t n_entries, const void* pool, const int32_t* order, const int32_t* offset, const float* score,
                           const void* d_out, float* d_pool, void* d_user, float* d_score, void* workspace, int64_t workspace_bytes,
                           void* stream)
{
    ckv_status st = check_gather(device, dtype, n, n_groups, head_dim, d_shared, n_entries);
    if (st != CKV_OK) return st;
    DeviceGuard dg(device);
    if (!dg.ok) return CKV_ERR_CUDA;
    const int e = dtype == CKV_F32 ? 4 : 2;
    const bool none = n == 0;
    if (!on_device(device, Arg{pool, e, !score}, Arg{order, 4, none}, Arg{offset, 4}, Arg{score, 4, true}, Arg{d_out, 16, none}, Arg{d_pool, 4},
                   Arg{d_user, e, true}, Arg{d_score, 4, none || !score}) ||
        (d_score && !score))
        return CKV_ERR_INVALID_ARG;
    st = check_workspace(device, workspace, workspace_bytes, segment_workspace(n, n_groups, head_dim));
    if (st != CKV_OK) return st;
    SegmentArgs a{};
    a.order = order;
    a.offset = offset;
    a.rows = d_out;
    a.stride = (int64_t)n_groups * head_dim;
    a.group_stride = head_dim;
    a.n = n;
    a.m = n_entries;
    a.G = n_groups;
    a.width = head_dim;
    a.skip = head_dim - d_shared;
    a.score = score;
    a.pool = score ? pool : nullptr;
    a.d_user = a.skip ? d_user : nullptr;
    a.d_score = d_score;
    a.sum = d_pool;
    return status_of(launch_segment_sum(dtype, a, workspace, (cudaStream_t)stream));
}

}  // extern "C"
