// Argument checks that the entry points share.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/e2ttt.h"

namespace e2ttt {

// Every workspace starts with a status block: word 0 is the device status of the last launch that used it.
constexpr size_t kStatusBytes = 256;

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_device();  // api.cu

// Lets a kernel have as much dynamic shared memory as its launches ask for, on the current device: asked for once per device, not at every
// launch (a decoder's launches take a few microseconds each), and always for the same amount, whichever host thread comes first.
constexpr int kMostSharedMemory = 226 * 1024;
template <auto KERNEL> cudaError_t allow_shared_memory() {
    static std::atomic<bool> granted[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const bool known = dev >= 0 && dev < 64;
    if (known && granted[dev].load(std::memory_order_acquire)) return cudaSuccess;
    e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSharedMemory);
    if (e == cudaSuccess && known) granted[dev].store(true, std::memory_order_release);
    return e;
}

}  // namespace e2ttt
