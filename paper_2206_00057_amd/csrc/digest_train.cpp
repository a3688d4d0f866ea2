// Host side of the operators that train normalised layers (layer norm): the
// checks of their arguments and their launches.  They belong to no partition
// handle.
#include "digest.h"
#include "status.h"
#include "train_kernels.h"

#include <hip/hip_runtime_api.h>

#include <cfloat>
#include <cmath>
#include <cstdint>

using digest::fail;
using digest::hip_check;

namespace {

constexpr size_t kAlign = 256;
constexpr int32_t kMaxWidth = 65536;

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

static_assert(DIGEST_F32 == digest::kF32 && DIGEST_BF16 == digest::kBF16 &&
                  DIGEST_F16 == digest::kF16,
              "the header's element types are the kernels'");

int elem_size(int32_t type) { return type == DIGEST_F32 ? 4 : 2; }

digest_status check_type(int32_t type)
{
    if (type != DIGEST_F32 && type != DIGEST_BF16 && type != DIGEST_F16)
        return fail(DIGEST_EINVAL, "unknown element type %d", type);
    return DIGEST_OK;
}

// The pointer is there and aligned to `align` bytes.
digest_status check_ptr(const void *p, size_t align, const char *name)
{
    if (!p)
        return fail(DIGEST_EINVAL, "%s is NULL", name);
    if ((uintptr_t)p % align)
        return fail(DIGEST_EINVAL, "%s is not %zu-byte aligned", name, align);
    return DIGEST_OK;
}

// A row-major array: the pointer, and its row stride in elements.
digest_status check_rows(const void *p, int64_t ld, int32_t width, int32_t type, const char *name)
{
    if (digest_status st = check_ptr(p, elem_size(type), name))
        return st;
    if (ld < width || ld > INT32_MAX)
        return fail(DIGEST_EINVAL, "row stride %lld of %s outside [%d, %d]", (long long)ld, name,
                    width, INT32_MAX);
    return DIGEST_OK;
}

digest_status check_workspace(const void *ws, size_t bytes, size_t need)
{
    if (digest_status st = check_ptr(ws, kAlign, "workspace"))
        return st;
    if (bytes < need)
        return fail(DIGEST_ENOMEM, "workspace of %zu bytes, %zu needed", bytes, need);
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

digest_status check_norm(int64_t n_rows, int32_t width)
{
    if (n_rows < 0 || n_rows >= INT32_MAX)
        return fail(DIGEST_EINVAL, "n_rows %lld out of range", (long long)n_rows);
    if (width < 1 || width > kMaxWidth)
        return fail(DIGEST_EINVAL, "width %d outside [1, %d]", width, kMaxWidth);
    return DIGEST_OK;
}

digest_status check_act(int32_t act)
{
    if (act != DIGEST_ACT_RELU && act != DIGEST_ACT_IDENTITY)
        return fail(DIGEST_EINVAL, "unknown activation %d", act);
    return DIGEST_OK;
}

size_t norm_workspace(int64_t n_rows, int32_t width)
{
    const size_t blocks = (size_t)digest::norm_partials((int32_t)n_rows, width);
    return align_up((blocks ? blocks : 1) * 2 * (size_t)width * sizeof(float));
}

}  // namespace

extern "C" {

digest_status digest_layer_norm_query(int64_t n_rows, int32_t width, size_t *workspace_bytes)
{
    if (digest_status st = check_norm(n_rows, width))
        return st;
    if (!workspace_bytes)
        return fail(DIGEST_EINVAL, "NULL output");
    *workspace_bytes = norm_workspace(n_rows, width);
    return DIGEST_OK;
}

digest_status digest_layer_norm_forward(int64_t n_rows, int32_t width, int32_t type,
                                        const void *x, int64_t ldx, const float *gain,
                                        const float *shift, float eps, int32_t act, void *y,
                                        int64_t ldy, float *stats, void *hip_stream)
{
    if (digest_status st = check_norm(n_rows, width))
        return st;
    if (digest_status st = check_type(type))
        return st;
    if (digest_status st = check_act(act))
        return st;
    if (!(eps >= FLT_MIN) || !std::isfinite(eps))
        return fail(DIGEST_EINVAL, "eps %g is not a positive normal number", (double)eps);
    if (n_rows == 0)
        return DIGEST_OK;
    if (digest_status st = check_rows(x, ldx, width, type, "x"))
        return st;
    if (digest_status st = check_rows(y, ldy, width, type, "y"))
        return st;
    if (gain)
        if (digest_status st = check_ptr(gain, 4, "gain"))
            return st;
    if (shift)
        if (digest_status st = check_ptr(shift, 4, "shift"))
            return st;
    if (stats)
        if (digest_status st = check_ptr(stats, 8, "stats"))
            return st;
    if (digest_status st = check_stream((hipStream_t)hip_stream))
        return st;
    return hip_check(digest::launch_norm_forward(type, (int32_t)n_rows, width, x, ldx, gain, shift,
                                                 eps, act == DIGEST_ACT_RELU, y, ldy, stats,
                                                 (hipStream_t)hip_stream),
                     "layer norm forward");
}

digest_status digest_layer_norm_backward(int64_t n_rows, int32_t width, int32_t type,
                                         const void *x, int64_t ldx, const float *gain,
                                         int32_t act, const void *y, int64_t ldy, const void *dy,
                                         int64_t lddy, const float *stats, void *dx, int64_t lddx,
                                         float *dgain, float *dshift, void *workspace,
                                         size_t bytes, void *hip_stream)
{
    if (digest_status st = check_norm(n_rows, width))
        return st;
    if (digest_status st = check_type(type))
        return st;
    if (digest_status st = check_act(act))
        return st;
    const bool relu = act == DIGEST_ACT_RELU;
    if (n_rows > 0) {
        if (digest_status st = check_rows(x, ldx, width, type, "x"))
            return st;
        if (digest_status st = check_rows(dy, lddy, width, type, "dy"))
            return st;
        if (relu)
            if (digest_status st = check_rows(y, ldy, width, type, "y"))
                return st;
        if (dx)
            if (digest_status st = check_rows(dx, lddx, width, type, "dx"))
                return st;
        if (digest_status st = check_ptr(stats, 8, "stats"))
            return st;
    }
    if (gain)
        if (digest_status st = check_ptr(gain, 4, "gain"))
            return st;
    if (dgain)
        if (digest_status st = check_ptr(dgain, 4, "dgain"))
            return st;
    if (dshift)
        if (digest_status st = check_ptr(dshift, 4, "dshift"))
            return st;
    if (dgain || dshift)
        if (digest_status st = check_workspace(workspace, bytes, norm_workspace(n_rows, width)))
            return st;
    if (digest_status st = check_stream((hipStream_t)hip_stream))
        return st;
    return hip_check(digest::launch_norm_backward(type, (int32_t)n_rows, width, x, ldx, gain, y,
                                                  ldy, dy, lddy, stats, relu, dx, lddx, dgain,
                                                  dshift, (float *)workspace,
                                                  (hipStream_t)hip_stream),
                     "layer norm backward");
}

}  // extern "C"
