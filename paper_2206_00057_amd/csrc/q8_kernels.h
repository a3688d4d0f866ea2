// Internal interface between the host code of the 8-bit rows (digest_q8.cpp,
// and digest_host.cpp for a partition's calls) and their gfx950 kernels
// (q8_kernels.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

#include "digest.h"

namespace digest {

// Codes of a row: d of them, zeros up to the next multiple of kQ8Align, rows a
// multiple of kQ8Align bytes apart.
constexpr int kQ8Align = 16;
constexpr int32_t q8_padded(int32_t d) { return (d + kQ8Align - 1) / kQ8Align * kQ8Align; }

// Row numbers: null (row i is number i), int64 of a caller's array, or int32
// of the library's own lists.
struct RowList {
    const void *p = nullptr;
    bool wide = false;
};

// Rows of `type` (the values of train_kernels.h), ldx elements apart: row
// src[i] < n_x becomes row dst[i] of the codes (ldq apart) and scales, i < n.
// A src[i] outside [0, n_x) gives a row of NaN; dst entries must be distinct
// and in range (the library's own).
hipError_t launch_quantize_rows(int32_t type, int32_t n, int32_t d, const void *x, int64_t ldx,
                                RowList src, int64_t n_x, int8_t *codes, int64_t ldq,
                                float *scales, RowList dst, hipStream_t s);
// The columns of a row-major rows x cols w as rows of codes.
hipError_t launch_quantize_columns(int32_t type, int32_t rows, int32_t cols, const void *w,
                                   int64_t ldw, int8_t *codes, int64_t ldq, float *scales,
                                   hipStream_t s);
// y[i] = the values of row src[i] < n_x of the codes; NaN if it is outside.
hipError_t launch_dequantize_rows(int32_t type, int32_t n, int32_t d, const int8_t *codes,
                                  int64_t ldq, const float *scales, RowList src, int64_t n_x,
                                  void *y, int64_t ldy, hipStream_t s);
// out[r] = sum over row r's entries of val scale codes[col] for the rows that
// the blocks name (as launch_spmm, the n_long long rows first); out is 16-byte
// aligned, its rows ldo apart, a multiple of 4 and at least d; the columns from
// d to the next multiple of 4 hold nothing that may be used (short rows' are
// written, long rows' are not).
struct SpmmBlock;
hipError_t launch_q8_aggregate(const SpmmBlock *blocks, int32_t n_blocks, int32_t n_long,
                               const int32_t *rowptr, const int32_t *col, const float *val,
                               const int8_t *codes, int64_t ldq, const float *scales, int32_t d,
                               float *out, int64_t ldo, hipStream_t s);
// y[r][j] = act(s_r t_j sum_c q[r][c] p[j][c]) over k columns of codes, k a
// multiple of kQ8Align and at most 65536.
hipError_t launch_q8_product(int32_t type, int32_t n, int32_t m, int32_t k, const int8_t *q,
                             int64_t ldq, const float *s, const int8_t *p, int64_t ldp,
                             const float *t, bool relu, void *y, int64_t ldy, hipStream_t st);
// dw[c][j] = sum_r q[r][c] s_r D[r][j], D = dy or dy 1[y > 0] (y not null);
// part holds q8_grad_floats floats.
size_t q8_grad_floats(int32_t n, int32_t k, int32_t m);
// Slices of the rows that it sums, for contiguous dy and y.
int32_t q8_grad_slices(int32_t n, int32_t k, int32_t m);
hipError_t launch_q8_weight_grad(int32_t type, int32_t n, int32_t k, int32_t m, const int8_t *q,
                                 int64_t ldq, const float *s, const void *dy, int64_t lddy,
                                 const void *y, int64_t ldy, float *part, float *dw,
                                 hipStream_t st);

// The launches that a partition's calls make, handed to them by digest_q8.cpp,
// so that digest_host.cpp links without the kernels of the 8-bit rows.
struct Q8Ops {
    decltype(&launch_quantize_rows) quantize;
    decltype(&launch_dequantize_rows) dequantize;
    decltype(&launch_q8_aggregate) aggregate;
    decltype(&launch_q8_product) product;
    decltype(&q8_grad_floats) grad_floats;
    decltype(&q8_grad_slices) grad_slices;
    decltype(&launch_q8_weight_grad) weight_grad;
};
digest_status partition_set_keep(digest_partition *p, int32_t mode, const Q8Ops *ops);
digest_status partition_push_q8(digest_partition *p, int32_t level, const float *h_own,
                                int8_t *codes, float *scales, int32_t mode, const Q8Ops &ops,
                                hipStream_t s);
digest_status partition_pull_q8(digest_partition *p, int32_t level, const int8_t *codes,
                                const float *scales, const Q8Ops &ops, hipStream_t s);
digest_status partition_forward_q8(digest_partition *p, int32_t layer, const float *h_in,
                                   const int8_t *w_codes, const float *w_scales, float *h_out,
                                   int32_t act, hipStream_t s);

}  // namespace digest
