// Device helpers shared by the kernel sources.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace digest {

constexpr int kWave = 64;

// The dispatcher deals workgroups to the 8 XCDs (each with its own L2) in
// turn by linear id.  xcd_contiguous maps the linear id p of an n-workgroup
// grid to a logical id such that every XCD receives one contiguous run of
// logical ids, in increasing order; it is a bijection of [0, n).  Kernels
// order their logical work so that neighbours share operand data.
constexpr uint32_t kXcds = 8;

__device__ __forceinline__ uint32_t xcd_contiguous(uint32_t p, uint32_t n)
{
    const uint32_t q = n / kXcds, rem = n % kXcds;
    const uint32_t x = p % kXcds, slot = p / kXcds;
    return (x < rem ? x * (q + 1) : rem * (q + 1) + (x - rem) * q) + slot;
}

// A workgroup barrier for data in LDS alone: __syncthreads() also waits for
// the global loads in flight, which are the next tiles.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

}  // namespace digest
