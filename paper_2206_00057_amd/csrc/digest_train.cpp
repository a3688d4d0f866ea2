// Host side of the operators that train normalised layers (layer norm, the
// orthogonalised update and the Muon update around it): the checks of their
// arguments, their workspace and their launches.  They belong to no
// partition handle.
#include "digest.h"
#include "status.h"
#include "train_kernels.h"

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>

using digest::fail;
using digest::hip_check;
using digest::OrthBatch;
using digest::OrthItem;
using digest::OrthStep;

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

// --- orthogonalised matrices ---

constexpr int32_t kMaxMatrices = 256;
constexpr int32_t kMaxSteps = 64;
// Newton-Schulz coefficients of the Muon optimiser (Jordan et al., 2024).
constexpr float kMuonCoeffs[3] = {3.4445f, -4.7750f, 2.0315f};

int32_t pad(int32_t x, int32_t to) { return (x + to - 1) / to * to; }

// Sizes of a matrix's planes; with a base address also where they lie.
// Returns the bytes they take.
size_t place(OrthItem &it, int32_t rows, int32_t cols, char *base)
{
    it.rows = rows, it.cols = cols;
    it.r = std::min(rows, cols), it.c = std::max(rows, cols);
    it.rp = it.rk = pad(it.r, digest::kOrthPad), it.cp = it.ck = pad(it.c, digest::kOrthPad);
    it.sums = (int32_t)std::min<int64_t>(
        digest::kOrthSumBlocks,
        ((int64_t)rows * cols + digest::kOrthSumRun - 1) / digest::kOrthSumRun);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *p = base ? base + at : nullptr;
        at += align_up(bytes);
        return p;
    };
    it.part = (double *)take(sizeof(double) * digest::kOrthSumBlocks);
    it.X = (uint16_t *)take((size_t)4 * it.rp * it.ck);
    it.Xt[0] = (uint16_t *)take((size_t)4 * it.cp * it.rk);
    it.Xt[1] = (uint16_t *)take((size_t)4 * it.cp * it.rk);
    it.A = (uint16_t *)take((size_t)4 * it.rp * it.rk);
    it.B = (uint16_t *)take((size_t)4 * it.rp * it.rk);
    return at;
}

digest_status check_matrices(int32_t count, const int32_t *rows, const int32_t *cols)
{
    if (count < 1 || count > kMaxMatrices)
        return fail(DIGEST_EINVAL, "need 1 <= count <= %d, got %d", kMaxMatrices, count);
    if (!rows || !cols)
        return fail(DIGEST_EINVAL, "NULL rows or cols");
    for (int32_t i = 0; i < count; ++i)
        if (rows[i] < 1 || rows[i] > kMaxWidth || cols[i] < 1 || cols[i] > kMaxWidth)
            return fail(DIGEST_EINVAL, "matrix %d is %d x %d, sides outside [1, %d]", i, rows[i],
                        cols[i], kMaxWidth);
    return DIGEST_OK;
}

// The matrices run kOrthItems at a time, every group in the same memory.
size_t orth_workspace(int32_t count, const int32_t *rows, const int32_t *cols)
{
    size_t most = 0;
    for (int32_t i = 0; i < count; i += digest::kOrthItems) {
        OrthBatch b{};
        size_t bytes = 0;
        for (int32_t j = i; j < std::min(count, i + digest::kOrthItems); ++j)
            bytes += place(b.item[b.n++], rows[j], cols[j], nullptr);
        most = std::max(most, bytes + align_up(digest::orth_partials(b)));
    }
    return most;
}

// The steps' coefficients and scales.  Singular values of X_0 lie in [0, 1];
// those of a step's result are bounded by the largest |a x + b x^3 + c x^5| on
// the bounds before, and bound its elements; the same for A = X X^T and for
// B = a I + b A + c A^2, whose eigenvalues are a + b x^2 + c x^4.
digest_status plan_steps(int32_t steps, const float *coeffs, OrthStep *out)
{
    if (steps < 1 || steps > kMaxSteps)
        return fail(DIGEST_EINVAL, "need 1 <= steps <= %d, got %d", kMaxSteps, steps);
    auto exponent = [](double bound) { return (int32_t)std::floor(std::log2(64000.0 / bound)); };
    double s = 1.0;
    for (int32_t k = 0; k < steps; ++k) {
        const float *f = coeffs ? coeffs + 3 * k : kMuonCoeffs;
        const double a = f[0], b = f[1], c = f[2];
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c))
            return fail(DIGEST_EINVAL, "the coefficients of step %d are not finite", k);
        const double l = s * s;
        auto poly = [&](double y) { return std::fabs(a + b * y + c * y * y); };
        double q = std::max(poly(0), poly(l)), p = s * poly(l);
        if (c != 0 && -b / (2 * c) > 0 && -b / (2 * c) < l)
            q = std::max(q, poly(-b / (2 * c)));
        // extrema of the odd polynomial: a + 3 b y + 5 c y^2 = 0.  t is formed
        // without a difference, so that neither root is lost as c vanishes
        const double disc = 9 * b * b - 20 * a * c;
        double y[2] = {-1, -1};
        if (disc >= 0) {
            const double t = -0.5 * (3 * b + std::copysign(std::sqrt(disc), b));
            if (c != 0)
                y[0] = t / (5 * c);
            if (t != 0)
                y[1] = a / t;
        }
        for (double v : y)
            if (v > 0 && v < l)
                p = std::max(p, std::sqrt(v) * poly(v));
        constexpr double kRange = 1 << 20;
        if (!(p <= kRange) || !(p >= 1 / kRange) || !(q <= kRange) || !(q >= 1 / kRange))
            return fail(DIGEST_EINVAL,
                        "the coefficients of step %d take singular values of at most %g to at "
                        "most %g (bounds outside 2^-20 .. 2^20)", k, s, p);
        out[k] = OrthStep{f[0], f[1], f[2], exponent(s), exponent(l), exponent(q), exponent(p),
                          k & 1};
        s = p;
    }
    return DIGEST_OK;
}

// Every matrix of the group fits one workgroup's LDS.
bool whole(const OrthBatch &b, int32_t steps)
{
    for (int32_t i = 0; i < b.n; ++i)
        if (b.item[i].r > digest::kWholeRows || b.item[i].c > digest::kWholeCols)
            return false;
    return steps <= digest::kWholeSteps;
}

// From U (and, for larger matrices, its partial sums) to the result.
digest_status run_steps(const OrthBatch &batch, const OrthStep *plan, int32_t steps, bool muon,
                        int32_t type, float keep, void *partials, hipStream_t s)
{
    if (whole(batch, steps))
        return hip_check(
            digest::launch_orth_whole(batch, plan, steps, muon, type, keep, s),
            "orthogonalisation");
    if (!muon)
        if (digest_status st = hip_check(digest::launch_orth_sum(batch, type, s), "norm"))
            return st;
    if (digest_status st = hip_check(
            digest::launch_orth_split(batch, muon ? DIGEST_F32 : type, plan[0].ex, s), "split"))
        return st;
    return hip_check(digest::launch_orth_steps(batch, plan, steps, muon, type, keep,
                                               (float *)partials, s),
                     "orthogonalisation");
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
    if (x == y && ldx != ldy)
        return fail(DIGEST_EINVAL, "y is x with another row stride");
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
    if (n_rows > 0 && dx) {
        if (dx == dy && lddx != lddy)
            return fail(DIGEST_EINVAL, "dx is dy with another row stride");
        if (dx == x || (relu && dx == y))
            return fail(DIGEST_EINVAL, "dx is x or y");
    }
    if (dgain && dgain == dshift)
        return fail(DIGEST_EINVAL, "dgain is dshift");
    if (digest_status st = check_stream((hipStream_t)hip_stream))
        return st;
    return hip_check(digest::launch_norm_backward(type, (int32_t)n_rows, width, x, ldx, gain, y,
                                                  ldy, dy, lddy, stats, relu, dx, lddx, dgain,
                                                  dshift, (float *)workspace,
                                                  (hipStream_t)hip_stream),
                     "layer norm backward");
}

digest_status digest_orthogonalize_query(int32_t count, const int32_t *rows, const int32_t *cols,
                                         size_t *workspace_bytes)
{
    if (digest_status st = check_matrices(count, rows, cols))
        return st;
    if (!workspace_bytes)
        return fail(DIGEST_EINVAL, "NULL output");
    *workspace_bytes = orth_workspace(count, rows, cols);
    return DIGEST_OK;
}

digest_status digest_orthogonalize(int32_t count, const int32_t *rows, const int32_t *cols,
                                   int32_t type, const void *const *in, const int64_t *ld_in,
                                   void *const *out, const int64_t *ld_out, int32_t steps,
                                   const float *coeffs, void *workspace, size_t bytes,
                                   void *hip_stream)
{
    if (digest_status st = check_matrices(count, rows, cols))
        return st;
    if (digest_status st = check_type(type))
        return st;
    if (!in || !out)
        return fail(DIGEST_EINVAL, "NULL in or out");
    OrthStep plan[kMaxSteps];
    if (digest_status st = plan_steps(steps, coeffs, plan))
        return st;
    const void *order[kMaxMatrices];
    for (int32_t i = 0; i < count; ++i) {
        if (digest_status st = check_rows(in[i], ld_in ? ld_in[i] : cols[i], cols[i], type, "in"))
            return st;
        if (digest_status st =
                check_rows(out[i], ld_out ? ld_out[i] : cols[i], cols[i], type, "out"))
            return st;
        order[i] = out[i];
    }
    std::sort(order, order + count);
    for (int32_t i = 1; i < count; ++i)
        if (order[i] == order[i - 1])
            return fail(DIGEST_EINVAL, "two matrices have the same output");
    for (int32_t i = 0; i < count; ++i)
        if (in[i] != out[i] && std::binary_search(order, order + count, in[i]))
            return fail(DIGEST_EINVAL, "matrix %d is the output of another", i);
    if (digest_status st =
            check_workspace(workspace, bytes, orth_workspace(count, rows, cols)))
        return st;
    hipStream_t s = (hipStream_t)hip_stream;
    if (digest_status st = check_stream(s))
        return st;
    for (int32_t i0 = 0; i0 < count; i0 += digest::kOrthItems) {
        OrthBatch batch{};
        char *base = (char *)workspace;
        batch.n = std::min(count - i0, digest::kOrthItems);
        for (int32_t j = 0; j < batch.n; ++j) {
            const int32_t i = i0 + j;
            OrthItem &it = batch.item[j];
            base += place(it, rows[i], cols[i], base);
            it.u = in[i], it.ldu = ld_in ? ld_in[i] : cols[i];
            it.out = out[i], it.ldo = ld_out ? ld_out[i] : cols[i];
        }
        if (digest_status st = run_steps(batch, plan, steps, false, type, 0.f, base, s))
            return st;
    }
    return DIGEST_OK;
}

digest_status digest_muon_average(int32_t count, const int32_t *rows, const int32_t *cols,
                                  float *const *w, float *const *momentum,
                                  const float *const *grads, int32_t n_grads, float lr, float beta,
                                  float decay, const float *scales, int32_t nesterov,
                                  int32_t steps, const float *coeffs, void *workspace,
                                  size_t bytes, void *hip_stream)
{
    if (digest_status st = check_matrices(count, rows, cols))
        return st;
    if (n_grads < 1 || n_grads > 64)
        return fail(DIGEST_EINVAL, "need 1 <= n_grads <= 64, got %d", n_grads);
    if (!w || !momentum || !grads)
        return fail(DIGEST_EINVAL, "NULL w, momentum or grads");
    // the weights and momenta are replaced: no factor may make them NaN
    const float keep = 1.f - lr * decay;
    if (!std::isfinite(lr) || !std::isfinite(beta) || !std::isfinite(decay) ||
        !std::isfinite(keep))
        return fail(DIGEST_EINVAL, "lr %g, beta %g, decay %g or 1 - lr decay is not finite",
                    (double)lr, (double)beta, (double)decay);
    for (int32_t i = 0; scales && i < count; ++i)
        if (!std::isfinite(scales[i]) || !std::isfinite(lr * scales[i]))
            return fail(DIGEST_EINVAL, "scale %g of matrix %d, or lr times it, is not finite",
                        (double)scales[i], i);
    OrthStep plan[kMaxSteps];
    if (digest_status st = plan_steps(steps, coeffs, plan))
        return st;
    // what is written: weights and momenta, each range once
    struct Range {
        uintptr_t from, to;
    } wr[2 * kMaxMatrices];
    for (int32_t i = 0; i < count; ++i) {
        const uintptr_t n = (uintptr_t)rows[i] * cols[i] * sizeof(float);
        if (digest_status st = check_ptr(w[i], 4, "w"))
            return st;
        if (digest_status st = check_ptr(momentum[i], 4, "momentum"))
            return st;
        wr[2 * i] = {(uintptr_t)w[i], (uintptr_t)w[i] + n};
        wr[2 * i + 1] = {(uintptr_t)momentum[i], (uintptr_t)momentum[i] + n};
    }
    std::sort(wr, wr + 2 * count, [](const Range &x, const Range &y) { return x.from < y.from; });
    for (int32_t i = 1; i < 2 * count; ++i)
        if (wr[i].from < wr[i - 1].to)
            return fail(DIGEST_EINVAL, "weights and momenta overlap");
    for (int32_t i = 0; i < count; ++i)
        for (int32_t m = 0; m < n_grads; ++m) {
            const float *g = grads[(int64_t)i * n_grads + m];
            if (digest_status st = check_ptr(g, 4, "gradient"))
                return st;
            const uintptr_t from = (uintptr_t)g,
                            to = from + (uintptr_t)rows[i] * cols[i] * sizeof(float);
            const Range *r = std::upper_bound(
                wr, wr + 2 * count, from, [](uintptr_t v, const Range &x) { return v < x.to; });
            if (r != wr + 2 * count && r->from < to)
                return fail(DIGEST_EINVAL, "gradient %d of matrix %d overlaps a weight or momentum",
                            m, i);
        }
    if (digest_status st = check_workspace(workspace, bytes, orth_workspace(count, rows, cols)))
        return st;
    hipStream_t s = (hipStream_t)hip_stream;
    if (digest_status st = check_stream(s))
        return st;
    for (int32_t i0 = 0; i0 < count; i0 += digest::kOrthItems) {
        OrthBatch batch{};
        char *base = (char *)workspace;
        batch.n = std::min(count - i0, digest::kOrthItems);
        for (int32_t j = 0; j < batch.n; ++j) {
            const int32_t i = i0 + j;
            OrthItem &it = batch.item[j];
            base += place(it, rows[i], cols[i], base);
            // U lies where the first step will write X^T: it is read before
            it.u = it.Xt[1], it.ldu = cols[i];
            it.out = w[i], it.ldo = cols[i];
            it.mom = momentum[i];
            it.scale = lr * (scales ? scales[i] : 1.f);
        }
        // (the gradients' pointers of one launch)
        const int32_t most = digest::kOrthGrads / n_grads;
        for (int32_t j = 0; j < batch.n; j += most) {
            OrthBatch part{};
            digest::OrthGrads g{};
            part.n = std::min(batch.n - j, most);
            for (int32_t k = 0; k < part.n; ++k) {
                part.item[k] = batch.item[j + k];
                for (int32_t m = 0; m < n_grads; ++m)
                    g.g[k * n_grads + m] = grads[(int64_t)(i0 + j + k) * n_grads + m];
            }
            if (digest_status st = hip_check(
                    digest::launch_muon_momentum(part, g, n_grads, beta, nesterov != 0, s),
                    "momentum"))
                return st;
        }
        if (digest_status st =
                run_steps(batch, plan, steps, true, DIGEST_F32, keep, base, s))
            return st;
    }
    return DIGEST_OK;
}

}  // extern "C"
