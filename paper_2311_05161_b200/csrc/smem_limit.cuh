// Dynamic shared-memory limit of a kernel: host code only (needs no device compiler).
#pragma once

#include <cuda_runtime_api.h>

#include <atomic>
#include <mutex>

namespace w4a8 {

constexpr int kMaxDevices = 64;

// Raises a kernel's limit to `bytes` unless an earlier call on this device already set it at least that
// high (`raised`: one slot per device, an array per kernel instance).  Setting and noting are one step for other
// host threads: the attribute is set absolutely, so a smaller size set after a larger one would lower it.
inline cudaError_t raise_smem_limit(const void *kernel, int bytes, std::atomic<int> (&raised)[kMaxDevices])
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    if (raised[dev].load(std::memory_order_acquire) >= bytes) return cudaSuccess;
    static std::mutex one_at_a_time;
    std::lock_guard<std::mutex> lock(one_at_a_time);
    if (raised[dev].load(std::memory_order_relaxed) >= bytes) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) raised[dev].store(bytes, std::memory_order_release);
    return e;
}
template <typename... KArgs>
inline cudaError_t raise_smem_limit(void (*kernel)(KArgs...), int bytes, std::atomic<int> (&raised)[kMaxDevices])
{
    return raise_smem_limit(reinterpret_cast<const void *>(kernel), bytes, raised);
}

}  // namespace w4a8
