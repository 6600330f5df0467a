// Host side of the tile loads: tensor maps and shared-memory limits.
#pragma once

#include <atomic>
#include <cuda.h>

#include "attention.h"

namespace pss {
namespace seq {

// A driver function, looked up once; null where there is none.
void* driver_call(const char* name, std::atomic<void*>* found);

// The driver's encoder of tensor maps wants the device's context bound to the calling
// thread, which no runtime call may have done yet in a new one.
cudaError_t bind_context();

// A map of rows [tokens][heads][dim] whose boxes are 64 values of `heads_box`
// heads of `tokens_box` tokens, in the 128-byte swizzle; what lies outside the
// tensor reads as zero.  spare: any device memory, the address of an empty tensor.
cudaError_t tile_map(CUtensorMap* map, const Rows& r, int tokens, int heads, int dim,
                     int heads_box, int tokens_box, const void* spare);

// Raises a kernel's dynamic shared-memory limit, once per device.  least_registers:
// what a kernel that splits its registers among its warpgroups was counted with; built
// with fewer a thread it would wait for them for ever, so it is not launched then.
template <typename K>
cudaError_t allow_smem(K* kernel, int bytes, std::atomic<uint64_t>* ready,
                       int least_registers = 0) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (ready->load(std::memory_order_acquire) & bit) return cudaSuccess;
    if (least_registers > 0) {
        cudaFuncAttributes built;
        e = cudaFuncGetAttributes(&built, kernel);
        if (e != cudaSuccess) return e;
        if (built.numRegs < least_registers) return cudaErrorInvalidConfiguration;
    }
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) ready->fetch_or(bit, std::memory_order_release);
    return e;
}

}  // namespace seq
}  // namespace pss
