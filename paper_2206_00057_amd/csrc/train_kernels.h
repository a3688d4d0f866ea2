// Internal interface between the host code of the training operators
// (digest_train.cpp) and their gfx950 kernels (norm_kernels.hip,
// orth_kernels.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

namespace digest {

// Element types of caller arrays (the values of digest.h).
enum ElemType : int32_t { kF32 = 0, kBF16 = 1, kF16 = 2 };

// Layer norm over rows of d elements, row strides in elements.  stats (mean,
// 1/sqrt(var + eps) per row), gain and shift may be null.
hipError_t launch_norm_forward(int32_t type, int32_t n, int32_t d, const void *x, int64_t ldx,
                               const float *gain, const float *shift, float eps, bool relu,
                               void *y, int64_t ldy, float *stats, hipStream_t s);

// Its backward: dx (may be null), and unless dgain and dshift are both null
// their partial sums, one [2][d] block per workgroup in part, then the sums.
// norm_partials(n, d) workgroups run.
int32_t norm_partials(int32_t n, int32_t d);
hipError_t launch_norm_backward(int32_t type, int32_t n, int32_t d, const void *x, int64_t ldx,
                                const float *gain, const void *y, int64_t ldy, const void *dy,
                                int64_t lddy, const float *stats, bool relu, void *dx,
                                int64_t lddx, float *dgain, float *dshift, float *part,
                                hipStream_t s);

}  // namespace digest
