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

// Orthogonalised matrices: X_0 = U / |U|_F, then steps of
// X <- (a I + b A + c A^2) X with A = X X^T, for X wide (r <= c; a tall U is
// worked on as its transpose).  X, its transpose, A and B = a I + b A + c A^2
// lie in memory as split planes: each value times a power of two as the sum
// of two fp16, in the order in which the matrix instructions take them.  Rows
// and k are padded to kOrthPad, with zeros.
constexpr int kOrthItems = 16;       // matrices of one launch
constexpr int kOrthGrads = 192;      // gradients of one launch (arguments below 4 KB)
constexpr int kOrthPad = 64;
constexpr int kOrthSumBlocks = 1024;  // partial sums of |U|_F^2, at most
constexpr int64_t kOrthSumRun = 1024;

struct OrthItem {
    int32_t rows, cols;              // of U and of the result
    int32_t r, c, rp, cp, rk, ck;    // of X: sides, rows padded, k padded
    const void *u;                   // U: the caller's, or fp32 in the workspace (muon)
    void *out;                       // the result, or the weights (muon)
    int64_t ldu, ldo;
    float *mom;                      // muon: momentum, in place
    float scale;                     // muon: w <- keep w - scale O
    int32_t sums;                    // partial sums in part
    double *part;
    uint16_t *X, *Xt[2], *A, *B;
};
struct OrthBatch {
    int32_t n;
    OrthItem item[kOrthItems];
};
struct OrthGrads {
    const float *g[kOrthGrads];      // item i: g[i * per_item ..]
};
// One step: its coefficients, and scale exponents (planes hold value * 2^e).
struct OrthStep {
    float a, b, c;
    int32_t ex, ea, eb, en;          // X, A, B, and X after the step
    int32_t from;                    // Xt[from] is read, Xt[from ^ 1] written
};
// part: sums of squares of U.
hipError_t launch_orth_sum(const OrthBatch &b, int32_t type, hipStream_t s);
// mom <- beta mom + g, u <- (nesterov ? g + beta mom : mom) with g the mean of
// the item's gradients, and part as above.
hipError_t launch_muon_momentum(const OrthBatch &b, const OrthGrads &g, int32_t per_item,
                                float beta, bool nesterov, hipStream_t s);
// X and Xt[0] from U: U / |U|_F * 2^e (zero for U = 0).
hipError_t launch_orth_split(const OrthBatch &b, int32_t type, int32_t e, hipStream_t s);
// Bytes of the steps' partial sums (joined), 16-byte aligned.
size_t orth_partials(const OrthBatch &b);
// Matrices that one workgroup holds in its LDS: everything from U (after
// launch_muon_momentum) to the result in one launch.
constexpr int kWholeRows = 64, kWholeCols = 256, kWholeSteps = 16;
hipError_t launch_orth_whole(const OrthBatch &b, const OrthStep *st, int32_t steps, bool muon,
                             int32_t type, float keep, hipStream_t s);
// The steps.  The result goes to out, as `type`, or (muon) into the weights:
// out <- keep out - scale O.
hipError_t launch_orth_steps(const OrthBatch &b, const OrthStep *steps, int32_t n, bool muon,
                             int32_t type, float keep, float *partials, hipStream_t s);

}  // namespace digest
