// One-time preparation of a kernel on a device.
#pragma once
#include <atomic>
#include <cuda_runtime.h>
#include <stdint.h>

namespace w2v {

// Lets kernel K use all the shared memory that its static share leaves, once per device; false if that fails or K was
// compiled with fewer than `regs` registers (kernels that move registers between warpgroups could then never do so).
template <auto K>
bool kernel_ready(int regs = 0)
{
    static std::atomic<uint64_t> done{0};
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess) return false;
    const uint64_t bit = 1ull << (device & 63);
    if (device < 64 && (done.load(std::memory_order_relaxed) & bit)) return true;
    cudaFuncAttributes at;
    if (cudaFuncGetAttributes(&at, K) != cudaSuccess || at.numRegs < regs) return false;
    if (cudaFuncSetAttribute(K, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - (int)at.sharedSizeBytes) != cudaSuccess) return false;
    if (device < 64) done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

}  // namespace w2v
