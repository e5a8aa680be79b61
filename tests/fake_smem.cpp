// The stand-in runtime with the permission that a launch with much shared memory needs: one number per kernel and process, as the real
// runtime keeps it, which any thread may set, lower values included.
#define cudaFuncSetAttribute any_size
#define cudaLaunchKernelExC any_launch
#include "fake_cudart.cpp"
#undef cudaFuncSetAttribute
#undef cudaLaunchKernelExC

namespace {
std::map<const void*, int> permitted;
void (*before_launch)() = nullptr;
}  // namespace

API void fake_before_launch(void (*hook)()) { before_launch = hook; }  // run once, when the next launch begins
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
