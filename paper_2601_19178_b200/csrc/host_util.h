// What the entry points share: the call's device made current for its time, and whose memory an argument points to.
#pragma once

#include <cuda_runtime.h>

namespace ckv {

struct DeviceGuard {
    int prev = -1;
    bool ok;
    explicit DeviceGuard(int dev)
    {
        ok = cudaGetDevice(&prev) == cudaSuccess;
        if (ok && prev != dev) ok = cudaSetDevice(dev) == cudaSuccess;
    }
    ~DeviceGuard()
    {
        int cur = -1;
        if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
    }
};

// Whose memory `p` points to: a device's (its ordinal), managed, or neither.
enum { kManagedMemory = -1, kNoDeviceMemory = -2 };
inline int memory_of(const void* p)
{
    cudaPointerAttributes at;
    if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
        cudaGetLastError();
        return kNoDeviceMemory;
    }
    return at.type == cudaMemoryTypeDevice ? at.device : at.type == cudaMemoryTypeManaged ? kManagedMemory : kNoDeviceMemory;
}
inline bool is_device_ptr(const void* p) { return memory_of(p) != kNoDeviceMemory; }

}  // namespace ckv
