// gfx950 kernels of the orthogonalised update (Newton-Schulz products) and of
// the Muon update around it.
//
// Small singular directions grow by the polynomial's slope at zero (3.4 a
// step), and rounding errors grow with them, so the products have to be as
// exact as fp32 ones.  The iterates are bounded (the singular values of X_0
// are at most 1, and the polynomial's maximum bounds those of every later
// one), so a fixed power of two takes them into fp16's range, where
//   2^e x = h + l,  h = fp16(2^e x),  l = fp16(2^e x - h)
// holds 22 to 23 bits of x, and of h h' + h l' + l h' + l l' the last, at
// most 2^-22 of a product and 2^-25 on average, is left out.  Three fp16
// matrix instructions then do the work of one fp32 product at 5 times the
// fp32 instructions' rate.  A and B are symmetric: only the tiles on and above
// the diagonal are computed, each stored twice.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "device.h"
#include "train_kernels.h"

namespace digest {
namespace {

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;
constexpr int kBlockK = 32;   // k of one line of a plane: 32 high, 32 low parts

// Offset (fp16) of k in a row of a plane; the low part lies kBlockK further.
__device__ __forceinline__ int64_t plane_at(int64_t row, int32_t pitch, int k)
{
    return row * 2 * pitch + (k / kBlockK) * (2 * kBlockK) + k % kBlockK;
}

// ---------------------------------------------------------------------------
// The update's matrix U and its norm
// ---------------------------------------------------------------------------

// The workgroup's sum of v, to all its threads, in a fixed order.
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double sum[kThreads / kWave];
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1)
        v += __shfl_xor(v, off);
    if (threadIdx.x % kWave == 0)
        sum[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < kThreads / kWave; ++w)
        v += sum[w];
    return v;
}

// Partial sums of the squares of U, 64 bits: their range holds the squares of
// every fp32 number.
template <class T>
__global__ __launch_bounds__(kThreads) void k_orth_sum(OrthBatch b)
{
    const OrthItem &it = b.item[blockIdx.y];
    if ((int)blockIdx.x >= it.sums)
        return;
    const T *u = (const T *)it.u;
    const int64_t n = (int64_t)it.rows * it.cols;
    double v = 0;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n;
         i += (int64_t)it.sums * kThreads) {
        const int64_t r = i / it.cols;
        const double x = (double)(float)u[r * it.ldu + (i - r * it.cols)];
        v += x * x;
    }
    v = block_sum(v);
    if (threadIdx.x == 0)
        it.part[blockIdx.x] = v;
}

__global__ __launch_bounds__(kThreads) void k_muon_momentum(OrthBatch b, OrthGrads grads,
                                                            int32_t per_item, float beta,
                                                            bool nesterov)
{
    const OrthItem &it = b.item[blockIdx.y];
    if ((int)blockIdx.x >= it.sums)
        return;
    const float *const *g = grads.g + blockIdx.y * per_item;
    float *u = (float *)it.u;
    const int64_t n = (int64_t)it.rows * it.cols;
    const float inv = 1.f / (float)per_item;
    double v = 0;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n;
         i += (int64_t)it.sums * kThreads) {
        float s = 0.f;
        for (int m = 0; m < per_item; ++m)
            s += g[m][i];
        s *= inv;
        const float mo = fmaf(beta, it.mom[i], s);
        it.mom[i] = mo;
        const float x = nesterov ? fmaf(beta, mo, s) : mo;
        u[i] = x;
        v += (double)x * (double)x;
    }
    v = block_sum(v);
    if (threadIdx.x == 0)
        it.part[blockIdx.x] = v;
}

// X_0 and its transpose as split planes.  A workgroup takes 64 x 64 of U: one
// plane has U's own layout (k along its columns), the other the transposed.
constexpr int kSplitTile = 64;

__device__ __forceinline__ void split8(const float (&x)[8], _Float16 *dst)
{
    half8 h, l;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        h[j] = (_Float16)x[j];
        l[j] = (_Float16)(x[j] - (float)h[j]);
    }
    *reinterpret_cast<half8 *>(dst) = h;
    *reinterpret_cast<half8 *>(dst + kBlockK) = l;
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_orth_split(OrthBatch b, double scale)
{
    __shared__ float tile[kSplitTile][kSplitTile + 1];
    const OrthItem &it = b.item[blockIdx.z];
    const bool tall = it.rows > it.cols;
    const int i0 = blockIdx.y * kSplitTile, j0 = blockIdx.x * kSplitTile;
    // padded extents of U's rows and columns
    if (i0 >= (tall ? it.cp : it.rp) || j0 >= (tall ? it.rp : it.cp))
        return;
    const double norm = sqrt(block_sum(threadIdx.x < it.sums ? it.part[threadIdx.x] : 0.0));
    const double f = norm == 0 ? 0.0 : scale / norm;
    const T *u = (const T *)it.u;
    const int tj = threadIdx.x % kSplitTile;
    for (int ti = threadIdx.x / kSplitTile; ti < kSplitTile; ti += kThreads / kSplitTile) {
        const int i = i0 + ti, j = j0 + tj;
        tile[ti][tj] = i < it.rows && j < it.cols
                           ? (float)((double)(float)u[(int64_t)i * it.ldu + j] * f)
                           : 0.f;
    }
    __syncthreads();
    _Float16 *p = (_Float16 *)(tall ? it.Xt[0] : it.X);
    _Float16 *pt = (_Float16 *)(tall ? it.X : it.Xt[0]);
    const int kp = tall ? it.rk : it.ck, kt = tall ? it.ck : it.rk;
    for (int q = threadIdx.x; q < kSplitTile * kSplitTile / 8; q += kThreads) {
        const int row = q / (kSplitTile / 8), k = q % (kSplitTile / 8) * 8;
        float x[8];
        if (j0 < kp) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = tile[row][k + e];
            split8(x, p + plane_at(i0 + row, kp, j0 + k));
        }
        if (i0 < kt) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = tile[k + e][row];
            split8(x, pt + plane_at(j0 + row, kt, i0 + k));
        }
    }
}

// ---------------------------------------------------------------------------
// Products of split planes
// ---------------------------------------------------------------------------

// D = P Q^T for planes P [M][K], Q [N][K] (both with k contiguous):
//   kGram    A  = X X^T             stored as planes, both halves
//   kPoly    B  = a I + b A + c A A stored as planes, both halves
//   kApply   X' = B X = B (X^T)^T   stored as planes of X' and of X'^T
//   kResult  the same into the caller's matrix
//   kUpdate  the same into the weights
enum OrthMode { kGram, kPoly, kApply, kResult, kUpdate };

constexpr int kBM = kOrthTile;                       // tile of D, both sides
constexpr int kWaveTile = kBM / 2;                   // 4 waves, 2 x 2
constexpr int kSub = kWaveTile / 32;                 // 32 x 32 blocks of a wave, each side
constexpr int kLine = 8;                             // 16-byte chunks of a line

struct OrthParams {
    float alpha;         // plane products to the stored value's scale
    float diag, lin;     // kPoly: a 2^eb, b 2^(eb - ea)
    float keep;
    int32_t from;
    int32_t tile0[kOrthItems + 1];
};

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

template <int MODE, class T>
__global__ __launch_bounds__(kThreads, 2) void k_orth_gemm(OrthBatch b, OrthParams pr)
{
    constexpr bool SYM = MODE == kGram || MODE == kPoly;
    // [row][chunk]: chunk j of row i holds the line's chunk j ^ (i & 7), so
    // that eight rows' reads of one chunk fall into different banks
    __shared__ half8 lds0[2][kBM * kLine], lds1[2][kBM * kLine];

    const uint32_t logical = xcd_contiguous(blockIdx.x, gridDim.x);
    int i = 0;
    while (i + 1 < b.n && (int)logical >= pr.tile0[i + 1])
        ++i;
    const OrthItem &it = b.item[i];
    int t = (int)logical - pr.tile0[i];
    int tm, tn;
    if constexpr (SYM) {
        // tiles on and above the diagonal, column by column
        tn = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
        while (tn * (tn + 1) / 2 > t)
            --tn;
        while ((tn + 1) * (tn + 2) / 2 <= t)
            ++tn;
        tm = t - tn * (tn + 1) / 2;
    } else {
        const int gm = it.rp / kBM;
        tm = t % gm;
        tn = t / gm;
    }
    const int K = MODE == kGram ? it.ck : it.rk;
    const half8 *P = reinterpret_cast<const half8 *>(MODE == kGram   ? it.X
                                                     : MODE == kPoly ? it.A
                                                                     : it.B) +
                     (int64_t)tm * kBM * (K / 4);
    const half8 *Q = reinterpret_cast<const half8 *>(MODE == kGram   ? it.X
                                                     : MODE == kPoly ? it.A
                                                                     : it.Xt[pr.from]) +
                     (int64_t)tn * kBM * (K / 4);
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int wm = wave / 2 * kWaveTile, wn = wave % 2 * kWaveTile;

    floatx16 acc[kSub][kSub];
#pragma unroll
    for (int x = 0; x < kSub; ++x)
#pragma unroll
        for (int y = 0; y < kSub; ++y)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                acc[x][y][e] = 0.f;

    // one line (32 k) of every row of both operands into LDS: a wave's
    // instruction takes 8 rows, 16 bytes a lane
    constexpr int kLoads = kBM / (8 * (kThreads / kWave));
    const int lrow = lane / kLine, chunk = (lane % kLine) ^ (lrow & 7);
    auto load = [&](int kb, half8 (*dst)[kBM * kLine]) {
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int row = (wave * kLoads + q) * 8;
            const int64_t at = (int64_t)(row + lrow) * (K / 4) + kb * kLine + chunk;
            __builtin_amdgcn_global_load_lds((global_void *)(P + at),
                                             (lds_void *)(&dst[0][row * kLine]), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((global_void *)(Q + at),
                                             (lds_void *)(&dst[1][row * kLine]), 16, 0, 0);
        }
    };
    auto multiply = [&](const half8 (*src)[kBM * kLine]) {
#pragma unroll
        for (int s = 0; s < kBlockK / 16; ++s) {
            half8 p[2][kSub], q[2][kSub];
            const int r = lane % 32;
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const int c = (4 * part + 2 * s + lane / 32) ^ (r & 7);
#pragma unroll
                for (int x = 0; x < kSub; ++x) {
                    p[part][x] = src[0][(wm + 32 * x + r) * kLine + c];
                    q[part][x] = src[1][(wn + 32 * x + r) * kLine + c];
                }
            }
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll
                for (int x = 0; x < kSub; ++x)
#pragma unroll
                    for (int y = 0; y < kSub; ++y)
                        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                            p[k == 2][x], q[k == 1][y], acc[x][y], 0, 0, 0);
        }
    };
    const int nk = K / kBlockK;   // even: k is padded to 64
    load(0, lds0);
    __syncthreads();
    for (int kb = 0; kb < nk; kb += 2) {
        load(kb + 1, lds1);
        multiply(lds0);
        __syncthreads();
        if (kb + 2 < nk)
            load(kb + 2, lds0);
        multiply(lds1);
        __syncthreads();
    }

    // element e of a lane: row 8 (e / 4) + 4 (lane / 32) + e % 4, column lane % 32
    // of its 32 x 32 block
#pragma unroll
    for (int x = 0; x < kSub; ++x)
#pragma unroll
        for (int y = 0; y < kSub; ++y) {
            const int mb = tm * kBM + wm + 32 * x, n = tn * kBM + wn + 32 * y + lane % 32;
            const int nb = n - lane % 32;
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const int m = mb + 8 * e4 + 4 * (lane / 32);
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = acc[x][y][4 * e4 + e] * pr.alpha;
                if constexpr (MODE == kPoly) {
                    const _Float16 *A = (const _Float16 *)it.A;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float l = 0.f;
                        if (nb < it.rk) {
                            const int64_t at = plane_at(m + e, it.rk, n);
                            l = (float)A[at] + (float)A[at + kBlockK];
                        }
                        v[e] = fmaf(l, pr.lin, v[e]) + (m + e == n ? pr.diag : 0.f);
                    }
                }
                if constexpr (MODE == kGram || MODE == kPoly || MODE == kApply) {
                    half4 h, l;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        h[e] = (_Float16)v[e];
                        l[e] = (_Float16)(v[e] - (float)h[e]);
                    }
                    _Float16 *d = (_Float16 *)(MODE == kGram ? it.A : MODE == kPoly ? it.B : it.X);
                    const int pitch = SYM ? it.rk : it.ck;
                    if (nb < pitch)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int64_t at = plane_at(m + e, pitch, n);
                            d[at] = h[e];
                            d[at + kBlockK] = l[e];
                        }
                    // the transposed: four consecutive k.  (A diagonal tile
                    // holds both halves itself.)
                    if ((!SYM || tm != tn) && mb < it.rk) {
                        _Float16 *dt = SYM ? d : (_Float16 *)it.Xt[pr.from ^ 1];
                        const int64_t at = plane_at(n, it.rk, m);
                        *reinterpret_cast<half4 *>(dt + at) = h;
                        *reinterpret_cast<half4 *>(dt + at + kBlockK) = l;
                    }
                } else {
                    const bool tall = it.rows > it.cols;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (m + e < it.r && n < it.c) {
                            const int64_t at = tall ? (int64_t)n * it.ldo + m + e
                                                    : (int64_t)(m + e) * it.ldo + n;
                            T *o = (T *)it.out + at;
                            if constexpr (MODE == kUpdate)
                                *o = (T)(pr.keep * (float)*o - it.scale * v[e]);
                            else
                                *o = (T)v[e];
                        }
                }
            }
        }
}

template <class F>
int32_t fill_tiles(const OrthBatch &b, OrthParams &pr, F tiles)
{
    pr.tile0[0] = 0;
    for (int i = 0; i < b.n; ++i)
        pr.tile0[i + 1] = pr.tile0[i] + tiles(b.item[i]);
    return pr.tile0[b.n];
}

template <int MODE, class T>
hipError_t gemm(const OrthBatch &b, OrthParams pr, hipStream_t s)
{
    const int32_t n = fill_tiles(b, pr, [](const OrthItem &it) {
        const int gm = it.rp / kBM, gn = it.cp / kBM;
        return MODE == kGram || MODE == kPoly ? gm * (gm + 1) / 2 : gm * gn;
    });
    k_orth_gemm<MODE, T><<<n, kThreads, 0, s>>>(b, pr);
    return hipGetLastError();
}

uint32_t most_sums(const OrthBatch &b)
{
    int32_t n = 1;
    for (int i = 0; i < b.n; ++i)
        n = std::max(n, b.item[i].sums);
    return (uint32_t)n;
}

}  // namespace

hipError_t launch_orth_sum(const OrthBatch &b, int32_t type, hipStream_t s)
{
    const dim3 grid(most_sums(b), b.n);
    switch (type) {
    case kF32: k_orth_sum<float><<<grid, kThreads, 0, s>>>(b); break;
    case kBF16: k_orth_sum<__bf16><<<grid, kThreads, 0, s>>>(b); break;
    case kF16: k_orth_sum<_Float16><<<grid, kThreads, 0, s>>>(b); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

hipError_t launch_muon_momentum(const OrthBatch &b, const OrthGrads &g, int32_t per_item,
                                float beta, bool nesterov, hipStream_t s)
{
    k_muon_momentum<<<dim3(most_sums(b), b.n), kThreads, 0, s>>>(b, g, per_item, beta, nesterov);
    return hipGetLastError();
}

hipError_t launch_orth_split(const OrthBatch &b, int32_t type, int32_t e, hipStream_t s)
{
    int32_t gi = 1, gj = 1;
    for (int i = 0; i < b.n; ++i) {
        const OrthItem &it = b.item[i];
        const bool tall = it.rows > it.cols;
        gi = std::max(gi, (tall ? it.cp : it.rp) / kSplitTile);
        gj = std::max(gj, (tall ? it.rp : it.cp) / kSplitTile);
    }
    const dim3 grid(gj, gi, b.n);
    const double scale = std::ldexp(1.0, e);
    switch (type) {
    case kF32: k_orth_split<float><<<grid, kThreads, 0, s>>>(b, scale); break;
    case kBF16: k_orth_split<__bf16><<<grid, kThreads, 0, s>>>(b, scale); break;
    case kF16: k_orth_split<_Float16><<<grid, kThreads, 0, s>>>(b, scale); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

hipError_t launch_orth_step(const OrthBatch &b, const OrthStep &st, bool last, bool muon,
                            int32_t type, float keep, hipStream_t s)
{
    OrthParams pr{};
    pr.keep = keep;
    pr.from = st.from;
    pr.alpha = std::ldexp(1.f, st.ea - 2 * st.ex);
    if (hipError_t e = gemm<kGram, float>(b, pr, s))
        return e;
    pr.alpha = std::ldexp(st.c, st.eb - 2 * st.ea);
    pr.lin = std::ldexp(st.b, st.eb - st.ea);
    pr.diag = std::ldexp(st.a, st.eb);
    if (hipError_t e = gemm<kPoly, float>(b, pr, s))
        return e;
    pr.alpha = std::ldexp(1.f, (last ? 0 : st.en) - st.eb - st.ex);
    if (!last)
        return gemm<kApply, float>(b, pr, s);
    if (muon)
        return gemm<kUpdate, float>(b, pr, s);
    switch (type) {
    case kF32: return gemm<kResult, float>(b, pr, s);
    case kBF16: return gemm<kResult, __bf16>(b, pr, s);
    case kF16: return gemm<kResult, _Float16>(b, pr, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace digest
