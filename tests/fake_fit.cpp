// The stand-in runtime with two devices, memory of either, and the permission that a launch with much shared memory needs: one number per
// kernel and process, as the real runtime keeps it, which any thread may set, lower values included.
#define cudaFuncSetAttribute any_size
#define cudaLaunchKernelExC any_launch
#define cudaPointerGetAttributes any_attributes
#include "fake_cudart.cpp"
#undef cudaFuncSetAttribute
#undef cudaLaunchKernelExC
#undef cudaPointerGetAttributes

namespace {
std::map<const void*, int> permitted;
std::map<const void*, int> kinds;  // of a block: the device, -1 for managed memory; else device 0
void (*before_launch)() = nullptr;
}  // namespace

API void fake_before_launch(void (*hook)()) { before_launch = hook; }  // run once, when the next launch begins
API void fake_block_of(void* block, int device) { kinds[block] = device; }
API cudaError_t cudaPointerGetAttributes(cudaPointerAttributes* a, const void* p)
{
    const cudaError_t e = any_attributes(a, p);
    const auto it = kinds.find(p);
    if (e == cudaSuccess && it != kinds.end()) {
        a->device = it->second < 0 ? 0 : it->second;
        if (it->second < 0) a->type = cudaMemoryTypeManaged;
    }
    return e;
}
API cudaError_t cudaFuncSetAttribute(const void* fn, cudaFuncAttribute, int v)
{
    std::lock_guard<std::mutex> lock(mu);
    permitted[fn] = v;
    return cudaSuccess;
}
API cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* fn, void** args)
{
    if (auto hook = before_launch) {
        before_launch = nullptr;
        hook();
    }
    {
        std::lock_guard<std::mutex> lock(mu);
        auto it = permitted.find(fn);
        if ((long)c->dynamicSmemBytes > (it == permitted.end() ? 48 * 1024 : it->second)) return cudaErrorInvalidValue;
    }
    return any_launch(c, fn, args);
}
