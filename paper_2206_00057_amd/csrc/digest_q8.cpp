// Host side of the rows held in 8 bits: the checks of their calls' arguments
// and their launches.
#include "digest.h"
#include "q8_kernels.h"
#include "status.h"

#include <hip/hip_runtime_api.h>

#include <cstdint>

using digest::fail;
using digest::hip_check;
using digest::RowList;

namespace {

constexpr size_t kAlign = 256;
constexpr int32_t kMaxWidth = 65536;

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

static_assert(DIGEST_Q8_STRIDE(1) == digest::q8_padded(1) &&
                  DIGEST_Q8_STRIDE(48) == digest::q8_padded(48),
              "the header's row stride is the kernels'");

int elem_size(int32_t type) { return type == DIGEST_F32 ? 4 : 2; }

digest_status check_type(int32_t type)
{
    if (type != DIGEST_F32 && type != DIGEST_BF16 && type != DIGEST_F16)
        return fail(DIGEST_EINVAL, "unknown element type %d", type);
    return DIGEST_OK;
}

digest_status check_act(int32_t act)
{
    if (act != DIGEST_ACT_RELU && act != DIGEST_ACT_IDENTITY)
        return fail(DIGEST_EINVAL, "unknown activation %d", act);
    return DIGEST_OK;
}

digest_status check_count(int64_t n, const char *name)
{
    if (n < 0 || n >= INT32_MAX)
        return fail(DIGEST_EINVAL, "%s %lld out of range", name, (long long)n);
    return DIGEST_OK;
}

digest_status check_width(int32_t d, const char *name)
{
    if (d < 1 || d > kMaxWidth)
        return fail(DIGEST_EINVAL, "%s %d outside [1, %d]", name, d, kMaxWidth);
    return DIGEST_OK;
}

// What a call reads or writes: named, so that overlaps are told.
struct Span {
    const char *name;
    const void *p;
    size_t bytes;
    bool out;
};

// The pointer is there and aligned to `align` bytes.
digest_status check_ptr(const void *p, size_t align, const char *name)
{
    if (!p)
        return fail(DIGEST_EINVAL, "%s is NULL", name);
    if ((uintptr_t)p % align)
        return fail(DIGEST_EINVAL, "%s is not %zu-byte aligned", name, align);
    return DIGEST_OK;
}

// Rows of elements, ld apart.
digest_status check_rows(const void *p, int64_t ld, int32_t width, int32_t type, const char *name)
{
    if (digest_status st = check_ptr(p, elem_size(type), name))
        return st;
    if (ld < width || ld > INT32_MAX)
        return fail(DIGEST_EINVAL, "row stride %lld of %s outside [%d, %d]", (long long)ld, name,
                    width, INT32_MAX);
    return DIGEST_OK;
}

// Rows of codes and their scales.
digest_status check_codes(const int8_t *codes, int64_t ld, int32_t width, const float *scales,
                          const char *name)
{
    if (digest_status st = check_ptr(codes, digest::kQ8Align, name))
        return st;
    if (ld < digest::q8_padded(width) || ld > INT32_MAX || ld % digest::kQ8Align)
        return fail(DIGEST_EINVAL, "row stride %lld of %s is no multiple of %d in [%d, %d]",
                    (long long)ld, name, digest::kQ8Align, digest::q8_padded(width), INT32_MAX);
    return check_ptr(scales, 4, "scales");
}

// Bytes from the first row's start to the last one's end.
size_t extent(int64_t n, int64_t ld, int64_t width, int size)
{
    return n > 0 ? ((size_t)(n - 1) * (size_t)ld + (size_t)width) * size : 0;
}

// No output shares memory with anything else of the call.
template <size_t N>
digest_status check_apart(const Span (&spans)[N])
{
    for (size_t i = 0; i < N; ++i)
        for (size_t j = 0; j < N; ++j) {
            const Span &a = spans[i], &b = spans[j];
            if (i == j || !a.out || !a.bytes || !b.bytes)
                continue;
            const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
            if (x < y + b.bytes && y < x + a.bytes)
                return fail(DIGEST_EINVAL, "%s overlaps %s", a.name, b.name);
        }
    return DIGEST_OK;
}

// The stream is one of the current device's (kernels run there).
digest_status check_stream(hipStream_t s)
{
    if (!s)
        return DIGEST_OK;
    int dev = -1;
    if (digest_status st = hip_check(hipGetDevice(&dev), "current device"))
        return st;
    hipDevice_t sdev = -1;
    if (digest_status st = hip_check(hipStreamGetDevice(s, &sdev), "stream device"))
        return st;
    if (sdev != dev)
        return fail(DIGEST_EINVAL, "the stream belongs to device %d, the current device is %d",
                    (int)sdev, dev);
    return DIGEST_OK;
}

// A list of rows of an array that has n_x of them.
digest_status check_list(const int64_t *rows, int64_t n_x, const char *name)
{
    if (!rows)
        return DIGEST_OK;
    if (digest_status st = check_count(n_x, name))
        return st;
    return check_ptr(rows, 8, "rows");
}

digest_status check_grad(int64_t n_rows, int32_t d_in, int32_t d_out)
{
    if (digest_status st = check_count(n_rows, "n_rows"))
        return st;
    if (digest_status st = check_width(d_in, "d_in"))
        return st;
    return check_width(d_out, "d_out");
}

size_t grad_workspace(int64_t n_rows, int32_t d_in, int32_t d_out)
{
    const size_t floats = digest::q8_grad_floats((int32_t)n_rows, d_in, d_out);
    return align_up(floats ? floats * sizeof(float) : 1);
}

constexpr digest::Q8Ops kOps = {digest::launch_quantize_rows, digest::launch_dequantize_rows,
                                digest::launch_q8_aggregate, digest::launch_q8_product,
                                digest::q8_grad_floats, digest::q8_grad_slices,
                                digest::launch_q8_weight_grad};

}  // namespace

extern "C" {

digest_status digest_partition_set_keep_mode(digest_partition *p, int32_t mode)
{
    return digest::partition_set_keep(p, mode, &kOps);
}

digest_status digest_push_q8(digest_partition *p, int32_t level, const float *h_own,
                             int8_t *codes, float *scales, int32_t mode, void *hip_stream)
{
    return digest::partition_push_q8(p, level, h_own, codes, scales, mode, kOps,
                                     (hipStream_t)hip_stream);
}

digest_status digest_pull_q8(digest_partition *p, int32_t level, const int8_t *codes,
                             const float *scales, void *hip_stream)
{
    return digest::partition_pull_q8(p, level, codes, scales, kOps, (hipStream_t)hip_stream);
}

digest_status digest_layer_forward_q8(digest_partition *p, int32_t layer, const float *h_in,
                                      const int8_t *w_codes, const float *w_scales, float *h_out,
                                      int32_t act, void *hip_stream)
{
    return digest::partition_forward_q8(p, layer, h_in, w_codes, w_scales, h_out, act,
                                        (hipStream_t)hip_stream);
}

digest_status digest_quantize_rows(int64_t n_rows, int32_t width, int32_t type, const void *x,
                                   int64_t ldx, const int64_t *rows, int64_t n_x, int8_t *codes,
                                   int64_t ldq, float *scales, void *hip_stream)
{
    if (digest_status st = check_count(n_rows, "n_rows"))
        return st;
    if (digest_status st = check_width(width, "width"))
        return st;
    if (digest_status st = check_type(type))
        return st;
    if (n_rows == 0)
        return DIGEST_OK;
    if (digest_status st = check_rows(x, ldx, width, type, "x"))
        return st;
    if (digest_status st = check_list(rows, n_x, "n_x"))
        return st;
    if (digest_status st = check_codes(codes, ldq, width, scales, "codes"))
        return st;
    const Span spans[] = {
        {"codes", codes, extent(n_rows, ldq, digest::q8_padded(width), 1), true},
        {"scales", scales, (size_t)n_rows * 4, true},
        {"x", x, extent(rows ? n_x : n_rows, ldx, width, elem_size(type)), false},
        {"rows", rows, rows ? (size_t)n_rows * 8 : 0, false}};
    if (digest_status st = check_apart(spans))
        return st;
    if (digest_status st = check_stream((hipStream_t)hip_stream))
        return st;
    return hip_check(digest::launch_quantize_rows(type, (int32_t)n_rows, width, x, ldx,
                                                  RowList{rows, true}, n_x, codes, ldq, scales,
                                                  RowList{}, (hipStream_t)hip_stream),
                     "quantize rows");
}

digest_status digest_quantize_columns(int32_t n_rows, int32_t n_cols, int32_t type, const void *w,
                                      int64_t ldw, int8_t *codes, int64_t ldq, float *scales,
                                      void *hip_stream)
{
    if (digest_status st = check_width(n_rows, "n_rows"))
        return st;
    if (digest_status st = check_width(n_cols, "n_cols"))
        return st;
    if (digest_status st = check_type(type))
        return st;
    if (digest_status st = check_rows(w, ldw, n_cols, type, "w"))
        return st;
    if (digest_status st = check_codes(codes, ldq, n_rows, scales, "codes"))
        return st;
    const Span spans[] = {
        {"codes", codes, extent(n_cols, ldq, digest::q8_padded(n_rows), 1), true},
        {"scales", scales, (size_t)n_cols * 4, true},
        {"w", w, extent(n_rows, ldw, n_cols, elem_size(type)), false}};
    if (digest_status st = check_apart(spans))
        return st;
    if (digest_status st = check_stream((hipStream_t)hip_stream))
        return st;
    return hip_check(digest::launch_quantize_columns(type, n_rows, n_cols, w, ldw, codes, ldq,
                                                     scales, (hipStream_t)hip_stream),
                     "quantize columns");
}

digest_status digest_dequantize_rows(int64_t n_rows, int32_t width, const int8_t *codes,
                                     int64_t ldq, const float *scales, const int64_t *rows,
                                     int64_t n_codes, int32_t type, void *y, int64_t ldy,
                                     void *hip_stream)
{
    if (digest_status st = check_count(n_rows, "n_rows"))
        return st;
    if (digest_status st = check_width(width, "width"))
        return st;
    if (digest_status st = check_type(type))
        return st;
    if (n_rows == 0)
        return DIGEST_OK;
    if (digest_status st = check_codes(codes, ldq, width, scales, "codes"))
        return st;
    if (digest_status st = check_list(rows, n_codes, "n_codes"))
        return st;
    if (digest_status st = check_rows(y, ldy, width, type, "y"))
        return st;
    const int64_t n = rows ? n_codes : n_rows;
    const Span spans[] = {
        {"y", y, extent(n_rows, ldy, width, elem_size(type)), true},
        {"codes", codes, extent(n, ldq, digest::q8_padded(width), 1), false},
        {"scales", scales, (size_t)n * 4, false},
        {"rows", rows, rows ? (size_t)n_rows * 8 : 0, false}};
    if (digest_status st = check_apart(spans))
        return st;
    if (digest_status st = check_stream((hipStream_t)hip_stream))
        return st;
    return hip_check(digest::launch_dequantize_rows(type, (int32_t)n_rows, width, codes, ldq,
                                                    scales, RowList{rows, true}, n_codes, y, ldy,
                                                    (hipStream_t)hip_stream),
                     "dequantize rows");
}

digest_status digest_q8_product(int64_t n_rows, int32_t d_in, int32_t d_out, const int8_t *codes,
                                int64_t ldq, const float *scales, const int8_t *w_codes,
                                int64_t ldw, const float *w_scales, int32_t act, int32_t type,
                                void *y, int64_t ldy, void *hip_stream)
{
    if (digest_status st = check_grad(n_rows, d_in, d_out))
        return st;
    if (digest_status st = check_type(type))
        return st;
    if (digest_status st = check_act(act))
        return st;
    if (n_rows == 0)
        return DIGEST_OK;
    if (digest_status st = check_codes(codes, ldq, d_in, scales, "codes"))
        return st;
    if (digest_status st = check_codes(w_codes, ldw, d_in, w_scales, "w_codes"))
        return st;
    if (digest_status st = check_rows(y, ldy, d_out, type, "y"))
        return st;
    const int32_t k = digest::q8_padded(d_in);
    const Span spans[] = {{"y", y, extent(n_rows, ldy, d_out, elem_size(type)), true},
                          {"codes", codes, extent(n_rows, ldq, k, 1), false},
                          {"scales", scales, (size_t)n_rows * 4, false},
                          {"w_codes", w_codes, extent(d_out, ldw, k, 1), false},
                          {"w_scales", w_scales, (size_t)d_out * 4, false}};
    if (digest_status st = check_apart(spans))
        return st;
    if (digest_status st = check_stream((hipStream_t)hip_stream))
        return st;
    return hip_check(digest::launch_q8_product(type, (int32_t)n_rows, d_out, k, codes, ldq, scales,
                                               w_codes, ldw, w_scales, act == DIGEST_ACT_RELU, y,
                                               ldy, (hipStream_t)hip_stream),
                     "product of 8-bit rows");
}

digest_status digest_q8_weight_grad_query(int64_t n_rows, int32_t d_in, int32_t d_out,
                                          size_t *workspace_bytes)
{
    if (digest_status st = check_grad(n_rows, d_in, d_out))
        return st;
    if (!workspace_bytes)
        return fail(DIGEST_EINVAL, "NULL output");
    *workspace_bytes = grad_workspace(n_rows, d_in, d_out);
    return DIGEST_OK;
}

digest_status digest_q8_weight_grad(int64_t n_rows, int32_t d_in, int32_t d_out,
                                    const int8_t *codes, int64_t ldq, const float *scales,
                                    int32_t type, const void *dy, int64_t lddy, int32_t act,
                                    const void *y, int64_t ldy, float *dw, void *workspace,
                                    size_t bytes, void *hip_stream)
{
    if (digest_status st = check_grad(n_rows, d_in, d_out))
        return st;
    if (digest_status st = check_type(type))
        return st;
    if (digest_status st = check_act(act))
        return st;
    const bool relu = act == DIGEST_ACT_RELU;
    if (n_rows > 0) {
        if (digest_status st = check_codes(codes, ldq, d_in, scales, "codes"))
            return st;
        if (digest_status st = check_rows(dy, lddy, d_out, type, "dy"))
            return st;
        if (relu)
            if (digest_status st = check_rows(y, ldy, d_out, type, "y"))
                return st;
    }
    if (digest_status st = check_ptr(dw, 4, "dw"))
        return st;
    if (digest_status st = check_ptr(workspace, kAlign, "workspace"))
        return st;
    const size_t need = grad_workspace(n_rows, d_in, d_out);
    if (bytes < need)
        return fail(DIGEST_ENOMEM, "workspace of %zu bytes, %zu needed", bytes, need);
    const Span spans[] = {
        {"dw", dw, (size_t)d_in * d_out * 4, true},
        {"workspace", workspace, need, true},
        {"codes", codes, extent(n_rows, ldq, digest::q8_padded(d_in), 1), false},
        {"scales", scales, (size_t)n_rows * 4, false},
        {"dy", dy, extent(n_rows, lddy, d_out, elem_size(type)), false},
        {"y", y, relu ? extent(n_rows, ldy, d_out, elem_size(type)) : 0, false}};
    if (digest_status st = check_apart(spans))
        return st;
    if (digest_status st = check_stream((hipStream_t)hip_stream))
        return st;
    return hip_check(digest::launch_q8_weight_grad(
                         type, (int32_t)n_rows, d_in, d_out, codes, ldq, scales, dy, lddy,
                         relu ? y : nullptr, ldy, (float *)workspace, dw,
                         (hipStream_t)hip_stream),
                     "weight gradient of 8-bit rows");
}

}  // extern "C"
