// gfx950 kernels of rows held in 8 bits: a scale and whole numbers of -127 to
// 127 for each row.  Writing and reading such rows, the product of two sets of
// them, and the weight gradient from kept ones.
//
// The scale is s = fl(a / 127) for the row's largest magnitude a, and the code
// of x the whole number nearest to the exact quotient x / s (ties to even), so
// that a row has one set of codes whatever computes them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "device.h"
#include "kernels.h"
#include "q8_kernels.h"
#include "train_kernels.h"

namespace digest {
namespace {

constexpr int kThreads = 256;

template <class T>
constexpr int kVecOf = 16 / (int)sizeof(T);

// A vector of N values of T, aligned to its elements only.
template <class T, int N>
struct Vec {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int64_t row_number(const RowList &l, int64_t i)
{
    if (!l.p)
        return i;
    return l.wide ? ((const int64_t *)l.p)[i] : ((const int32_t *)l.p)[i];
}

// v, a number in fp32, rounded to T.  (Without the barrier the compiler folds a
// product into the conversion to fp16, which then rounds it once.)
template <class T>
__device__ __forceinline__ T rounded(float v)
{
    if constexpr (std::is_same<T, _Float16>::value)
        asm("" : "+v"(v));
    return (T)v;
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// A row's scale and what its codes are formed with, from the bits of its
// largest magnitude (a NaN's are above infinity's, that is above any number's).
struct Scale {
    float s, inv;
    __device__ __forceinline__ explicit Scale(uint32_t top)
    {
        s = __uint_as_float(top) / 127.f;
        // below the normal numbers the quotients have no reciprocal to start from
        if (s < FLT_MIN)
            s = 0.f;
        inv = s > 0.f ? 1.f / s : 0.f;
        if (top >= 0x7f800000u)
            s = __uint_as_float(0x7fc00000u), inv = 0.f;
    }
};

// The codes of the four values x as bytes.  x inv plus 1.5 * 2^23 has the
// rounded quotient in its low byte; it is off by one at most, where the
// quotient lies next to a half.  r = x - q s is exact there (a multiple of s's
// last place below s), so that 2 |r| > s, or a tie at an odd q, tells.
__device__ __forceinline__ uint32_t codes4(const float (&x)[4], const Scale &sc)
{
    constexpr float kMagic = 12582912.f;
    float u[4], r[4];
    bool near = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u[i] = __builtin_fmaf(x[i], sc.inv, kMagic);
        r[i] = __builtin_fmaf(-(u[i] - kMagic), sc.s, x[i]);
        near |= __builtin_fabsf(r[i]) + __builtin_fabsf(r[i]) >= sc.s;
    }
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        b[i] = __float_as_uint(u[i]);
    if (near && sc.inv > 0.f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float twice = __builtin_fabsf(r[i]) + __builtin_fabsf(r[i]);
            if (twice > sc.s || (twice == sc.s && (b[i] & 1)))
                b[i] += r[i] > 0.f ? 1 : -1;
        }
    }
    if (!(sc.inv > 0.f))
        return 0;
    return (b[0] & 255) | (b[1] & 255) << 8 | (b[2] & 255) << 16 | b[3] << 24;
}

// A row in the registers of GL lanes (WAVES == 1, 64 / GL rows a wave) or of
// WAVES waves of one workgroup, Q vectors of 16 bytes a lane: one reading of x,
// four 16-byte loads a lane under way, and few lanes to find the largest of.
// Bound by memory: 304,051 of 306,250 rows of 256 float32 82 to 99 us (3.9 to 4.7
// TB/s), 16,384 x 4,096 bfloat16 41 us (4.9 TB/s); 304,051 x 47 float32, whose
// rows start anywhere, 16 us.
template <class T, int GL, int Q, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? kThreads : WAVES * kWave) void k_quantize_rows(
    int32_t n, int32_t d, const T *__restrict__ x, int64_t ldx, RowList src, int64_t n_x,
    int8_t *__restrict__ codes, int64_t ldq, float *__restrict__ scales, RowList dst)
{
    constexpr int V = kVecOf<T>;
    constexpr int L = WAVES == 1 ? GL : WAVES * kWave;   // lanes of a row
    typedef typename Vec<T, V>::type vec;
    const int lane = threadIdx.x % L;
    const int64_t row = WAVES == 1 ? (int64_t)blockIdx.x * (kThreads / GL) + threadIdx.x / GL
                                   : (int64_t)blockIdx.x;
    const bool live = row < n;
    const int64_t from = live ? row_number(src, row) : 0;
    const bool there = live && from >= 0 && from < n_x;
    const T *xr = x + (there ? from * ldx : 0);

    vec v[Q];
    uint32_t top = there ? 0 : 0x7fc00000u;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int c = (q * L + lane) * V;
        if (there && c + V <= d) {
            v[q] = *reinterpret_cast<const vec *>(xr + c);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                v[q][j] = there && c + j < d ? xr[c + j] : (T)0.f;
        }
    }
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int j = 0; j < V; ++j)
            top = max(top, magnitude((float)v[q][j]));
#pragma unroll
    for (int m = (WAVES == 1 ? GL : kWave) / 2; m > 0; m /= 2)
        top = max(top, (uint32_t)__shfl_xor((int)top, m));
    if constexpr (WAVES > 1) {
        __shared__ uint32_t red[WAVES];
        if (lane % kWave == 0)
            red[lane / kWave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
            top = max(top, red[w]);
    }
    if (!live)
        return;
    const Scale sc(top);
    const int64_t to = row_number(dst, row);
    int8_t *out = codes + to * ldq;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int c = (q * L + lane) * V;
        if (c >= q8_padded(d))
            continue;
        uint32_t w[V / 4];
#pragma unroll
        for (int j = 0; j < V / 4; ++j) {
            const float f[4] = {(float)v[q][4 * j], (float)v[q][4 * j + 1],
                                (float)v[q][4 * j + 2], (float)v[q][4 * j + 3]};
            w[j] = codes4(f, sc);
        }
        if constexpr (V == 4)
            *reinterpret_cast<uint32_t *>(out + c) = w[0];
        else
            *reinterpret_cast<uint2 *>(out + c) = make_uint2(w[0], w[1]);
    }
    if (lane == 0)
        scales[to] = sc.s;
}

// Columns of w as rows of codes: a workgroup takes C columns, a thread P pieces
// of 16 rows of one of them, in registers (P > 0: one reading of w), or in two
// passes (P == 0, rows past 16 P kColThreads / C).  A piece is 16 bytes of codes.
// Bound by latency: 602 x 256 float32 4 us (17 with 256 threads and two passes).
// Large weights, a call: 4,096 x 4,096 float32 26 us (3.2 TB/s), bfloat16 32 (1.6:
// 32 bytes of each row a workgroup), 8,192 x 1,024 bfloat16 92 (0.3: two passes
// over 64 workgroups).
constexpr int kColThreads = 1024;
template <class T, int C, int P>
__global__ __launch_bounds__(kColThreads) void k_quantize_columns(
    int32_t rows, int32_t cols, const T *__restrict__ w, int64_t ldw, int8_t *__restrict__ codes,
    int64_t ldq, float *__restrict__ scales)
{
    constexpr int G = kColThreads / C, H = P ? P : 1;
    __shared__ uint32_t red[kColThreads / kWave][C];
    const int c = threadIdx.x % C, g = threadIdx.x / C;
    const int64_t col = (int64_t)blockIdx.x * C + c;
    const int32_t left = col < cols ? rows : 0;
    auto load = [&](int32_t r0, T (&f)[16]) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            f[i] = r0 + i < left ? w[(int64_t)(r0 + i) * ldw + col] : (T)0.f;
    };
    auto largest = [](uint32_t top, const T (&f)[16]) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            top = max(top, magnitude((float)f[i]));
        return top;
    };
    T f[H][16];
    uint32_t top = 0;
    if constexpr (P > 0) {
#pragma unroll
        for (int p = 0; p < P; ++p)
            load((p * G + g) * 16, f[p]);
#pragma unroll
        for (int p = 0; p < P; ++p)
            top = largest(top, f[p]);
    } else {
        for (int32_t r0 = g * 16; r0 < left; r0 += G * 16) {
            load(r0, f[0]);
            top = largest(top, f[0]);
        }
    }
#pragma unroll
    for (int m = kWave / 2; m >= C; m /= 2)
        top = max(top, (uint32_t)__shfl_xor((int)top, m));
    if (threadIdx.x % kWave < C)
        red[threadIdx.x / kWave][c] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kColThreads / kWave; ++i)
        top = max(top, red[i][c]);
    if (left == 0)
        return;
    const Scale sc(top);
    if (g == 0)
        scales[col] = sc.s;
    auto store = [&](int32_t r0, const T (&f)[16]) {
        if (r0 >= rows)
            return;
        uint32_t p[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x[4] = {(float)f[4 * j], (float)f[4 * j + 1], (float)f[4 * j + 2],
                                (float)f[4 * j + 3]};
            p[j] = codes4(x, sc);
        }
        *reinterpret_cast<uint4 *>(codes + col * ldq + r0) = make_uint4(p[0], p[1], p[2], p[3]);
    };
    if constexpr (P > 0) {
#pragma unroll
        for (int p = 0; p < P; ++p)
            store((p * G + g) * 16, f[p]);
    } else {
        for (int32_t r0 = g * 16; r0 < rows; r0 += G * 16) {
            load(r0, f[0]);
            store(r0, f[0]);
        }
    }
}

// Lanes and vectors as in k_quantize_rows, rows wider than their GL Q V columns
// in several turns.  Bound by memory: 304,051 x 256 float32 in any order 67 us (5.8
// TB/s, the codes partly from the Infinity Cache), 16,384 x 4,096 bfloat16 32 us;
// rows that are not whole vectors, 304,051 x 47, 31 us.  (A lane an element for
// them, so that each is stored as one run: 44 us.)
template <class T, int GL, int Q>
__global__ __launch_bounds__(kThreads) void k_dequantize_rows(
    int32_t n, int32_t d, const int8_t *__restrict__ codes, int64_t ldq,
    const float *__restrict__ scales, RowList src, int64_t n_x, T *__restrict__ y, int64_t ldy)
{
    constexpr int V = kVecOf<T>;
    typedef typename Vec<T, V>::type vec;
    const int lane = threadIdx.x % GL;
    const int64_t row = (int64_t)blockIdx.x * (kThreads / GL) + threadIdx.x / GL;
    if (row >= n)
        return;
    const int64_t from = row_number(src, row);
    const bool there = from >= 0 && from < n_x;
    const float s = there ? scales[from] : __uint_as_float(0x7fc00000u);
    const int8_t *q8 = codes + (there ? from * ldq : 0);
    T *yr = y + row * ldy;
    for (int32_t c0 = 0; c0 < d; c0 += GL * Q * V) {
        uint32_t w[Q][V / 4];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int c = c0 + (q * GL + lane) * V;
            const bool in = there && c < d;
            if constexpr (V == 4) {
                w[q][0] = in ? *reinterpret_cast<const uint32_t *>(q8 + c) : 0;
            } else {
                const uint2 t = in ? *reinterpret_cast<const uint2 *>(q8 + c) : make_uint2(0, 0);
                w[q][0] = t.x, w[q][1] = t.y;
            }
        }
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int c = c0 + (q * GL + lane) * V;
            vec out;
#pragma unroll
            for (int j = 0; j < V; ++j)
                out[j] = rounded<T>((float)(int8_t)(w[q][j / 4] >> (8 * (j % 4))) * s);
            if (c + V <= d) {
                *reinterpret_cast<vec *>(yr + c) = out;
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (c + j < d)
                        yr[c + j] = out[j];
            }
        }
    }
}

// Rows of a contiguous y that are not whole vectors, R rows (R d whole vectors) a
// workgroup: their codes come into LDS in pieces of 16 bytes and leave as whole
// vectors at whole vectors' places, which may hold the end of one row and the
// start of the next.  304,051 x 47 float32 in random order 22 us against 31 with
// vectors anywhere, bfloat16 20 / 25, 101 float32 44 / 52, 300,000 x 7 in order 5.7 /
// 7.6; 602 bfloat16 loses (54 / 44).
constexpr int kFlatBytes = 16384;
template <class T>
__global__ __launch_bounds__(kThreads) void k_dequantize_flat(
    int32_t n, int32_t d, int32_t R, const int8_t *__restrict__ codes, int64_t ldq,
    const float *__restrict__ scales, RowList src, int64_t n_x, T *__restrict__ y)
{
    constexpr int V = kVecOf<T>;
    typedef T vec __attribute__((ext_vector_type(V)));
    __shared__ i32x4 lq[kFlatBytes / 16];
    __shared__ float ls[kFlatBytes / 16];
    const int64_t first = (int64_t)blockIdx.x * R;
    const int rows = (int)min((int64_t)R, n - first), pieces = (d + 15) / 16;
    for (int t = threadIdx.x; t < rows * pieces; t += kThreads) {
        const int r = t / pieces, p = t % pieces;
        const int64_t from = row_number(src, first + r);
        const bool there = from >= 0 && from < n_x;
        const i32x4 zero = {0, 0, 0, 0};
        lq[t] = there ? *reinterpret_cast<const i32x4 *>(codes + from * ldq + p * 16) : zero;
        if (p == 0)
            ls[r] = there ? scales[from] : __uint_as_float(0x7fc00000u);
    }
    __syncthreads();
    const int8_t *bytes = reinterpret_cast<const int8_t *>(lq);
    const int pad = pieces * 16, total = rows * d;
    constexpr int STEP = kThreads * V;
    const int dr = STEP / d, dc = STEP % d;
    int r0 = threadIdx.x * V / d, c0 = threadIdx.x * V % d;
    T *out = y + first * d;
    for (int e = threadIdx.x * V; e < total; e += STEP) {
        int r = r0, c = c0;
        vec v;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (e + i < total)
                v[i] = rounded<T>((float)bytes[r * pad + c] * ls[r]);
            if (++c == d)
                c = 0, ++r;
        }
        if (e + V <= total) {
            *reinterpret_cast<vec *>(out + e) = v;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (e + i < total)
                    out[e + i] = v[i];
        }
        r0 += dr, c0 += dc;
        if (c0 >= d)
            c0 -= d, ++r0;
    }
}

// out[r] = sum over the entries e of row r of val[e] scale[col e] codes[col e]: a
// store's rows in 8 bits gathered into the sums that are wanted of them.  Bound
// by the latency of few random reads a row.  GL lanes take a row's 16 GL
// columns.  Short rows (the blocks' runs of at most 8): all of one by GL
// lanes, which first fetch GL entries with their scales at once and then the
// entries' codes, U under way.  304,051 rows of 256 columns with 7.5 entries each
// 208 us and 34 for the long ones (259 a call; from a float32 store 404; a wave a
// row with the entries dealt to its groups of lanes 492).
template <int GL>
__global__ __launch_bounds__(8 * GL) void k_q8_aggregate(
    const SpmmBlock *__restrict__ blocks, const int32_t *__restrict__ rowptr,
    const int32_t *__restrict__ col, const float *__restrict__ val,
    const int8_t *__restrict__ codes, int64_t ldq, const float *__restrict__ scales, int32_t d,
    float *__restrict__ out, int64_t ldo)
{
    constexpr int U = 4;
    const SpmmBlock blk = blocks[blockIdx.x];
    const int gl = threadIdx.x % GL, g = threadIdx.x / GL;
    if (g >= blk.nrows)
        return;
    const int32_t row = blk.row + g, k0 = rowptr[row], k1 = rowptr[row + 1];
    for (int32_t c0 = 0; c0 < d; c0 += GL * 16) {
        const int32_t c = c0 + gl * 16;
        float acc[16] = {};
        for (int32_t kb = k0; kb < k1; kb += GL) {
            const int32_t mine = kb + gl < k1 ? col[kb + gl] : 0;
            const float w_mine = kb + gl < k1 ? val[kb + gl] * scales[mine] : 0.f;
            const int count = min(GL, k1 - kb);
            for (int j = 0; j < count; j += U) {
                i32x4 q[U];
                float w[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int at = min(j + u, GL - 1);
                    const int64_t r = __shfl(mine, at, GL);
                    w[u] = __shfl(w_mine, at, GL);
                    const i32x4 zero = {0, 0, 0, 0};
                    q[u] = zero;
                    if (j + u >= count)
                        w[u] = 0.f;
                    else if (c < d)
                        q[u] = *reinterpret_cast<const i32x4 *>(codes + r * ldq + c);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        acc[i] = __builtin_fmaf(
                            w[u], (float)(int8_t)(q[u][i / 4] >> (8 * (i % 4))), acc[i]);
            }
        }
        // (rows of out are 16-byte aligned: d rounded up to 4 floats apart)
        float *o = out + row * ldo + c;
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            if (c + i < d)
                *reinterpret_cast<f32x4 *>(o + i) = f32x4{acc[i], acc[i + 1], acc[i + 2],
                                                          acc[i + 3]};
    }
}

// The long rows, a workgroup each: its waves a run of entries, GL lanes every
// 64 / GL-th of them; the lanes' groups' sums, then the waves', are added in their
// order.
template <int GL>
__global__ __launch_bounds__(kSpmmThreads) void k_q8_aggregate_long(
    const SpmmBlock *__restrict__ blocks, const int32_t *__restrict__ col,
    const float *__restrict__ val, const int8_t *__restrict__ codes, int64_t ldq,
    const float *__restrict__ scales, int32_t d, float *__restrict__ out, int64_t ldo)
{
    constexpr int W = kSpmmThreads / kWave, G = kWave / GL, U = 4;
    __shared__ float red[W][GL * 16];
    const SpmmBlock blk = blocks[blockIdx.x];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int gl = lane % GL, g = lane / GL;
    const int32_t each = (blk.ke - blk.kb + W - 1) / W;
    const int32_t k0 = min(blk.ke, blk.kb + wave * each), k1 = min(blk.ke, k0 + each);
    for (int32_t c0 = 0; c0 < d; c0 += GL * 16) {
        const int32_t c = c0 + gl * 16;
        float acc[16] = {};
        for (int32_t k = k0 + g; k < k1; k += G * U) {
            i32x4 q[U];
            float w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int32_t e = k + u * G;
                const i32x4 zero = {0, 0, 0, 0};
                w[u] = 0.f, q[u] = zero;
                if (e < k1) {
                    const int64_t r = col[e];
                    w[u] = val[e] * scales[r];
                    if (c < d)
                        q[u] = *reinterpret_cast<const i32x4 *>(codes + r * ldq + c);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    acc[i] = __builtin_fmaf(w[u], (float)(int8_t)(q[u][i / 4] >> (8 * (i % 4))),
                                            acc[i]);
        }
#pragma unroll
        for (int m = GL; m < kWave; m *= 2)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                acc[i] += __shfl_xor(acc[i], m);
        __syncthreads();
        if (g == 0)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                red[wave][gl * 16 + i] = acc[i];
        __syncthreads();
        for (int i = threadIdx.x; i < GL * 16 && c0 + i < d; i += kSpmmThreads) {
            float v = red[0][i];
#pragma unroll
            for (int w = 1; w < W; ++w)
                v += red[w][i];
            out[blk.row * ldo + c0 + i] = v;
        }
    }
}

// An element of the product from its exact sum.  The smaller scale first: a
// whole number times it is at least the smallest normal number, so that
// nothing is lost on the way to a result that can be held.
__device__ __forceinline__ float scaled(int sum, float s, float t)
{
    const bool less = s < t;
    return (float)sum * (less ? s : t) * (less ? t : s);
}

// ReLU that keeps a NaN.
__device__ __forceinline__ float relu_of(float v, bool relu) { return relu && v <= 0.f ? 0.f : v; }

// Outputs of N channels in a row of row r: scaled, activated, rounded, stored
// below channel m.
template <class T, int N>
__device__ __forceinline__ void store_row(const int (&sum)[N], float sr,
                                          const float *__restrict__ t, bool relu, int64_t j,
                                          int32_t m, T *__restrict__ yr)
{
    if (j + N <= m) {
        typename Vec<T, N>::type v;
#pragma unroll
        for (int e = 0; e < N; ++e)
            v[e] = rounded<T>(relu_of(scaled(sum[e], sr, t[j + e]), relu));
        *reinterpret_cast<typename Vec<T, N>::type *>(yr + j) = v;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (j + e < m)
                yr[j + e] = rounded<T>(relu_of(scaled(sum[e], sr, t[j + e]), relu));
    }
}

// Few rows: bound by reading the weight's codes, 16 MT channels and 16 NT rows a
// workgroup, its W waves a share of k each, straight from memory; the waves'
// sums, whole numbers, are added through LDS.  One row x 4,096 x 4,096 5.4 us (3.1
// TB/s: one wave's loads after another and the sum, for 3.3 at a copy's rate), 64
// rows 12.
template <class T, int MT, int NT, int W>
__global__ __launch_bounds__(W *kWave) void k_q8_few(int32_t n, int32_t m, int32_t k,
                                                     const int8_t *__restrict__ q, int64_t ldq,
                                                     const float *__restrict__ s,
                                                     const int8_t *__restrict__ p, int64_t ldp,
                                                     const float *__restrict__ t, bool relu,
                                                     T *__restrict__ y, int64_t ldy)
{
    __shared__ i32x4 red[W][MT * NT][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int l = lane % 16, g = lane / 16;
    const int64_t j0 = (int64_t)blockIdx.x * (16 * MT), r0 = (int64_t)blockIdx.y * (16 * NT);
    const i32x4 zero = {0, 0, 0, 0};
    const int8_t *pj[MT], *qr[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
        pj[i] = p + min(j0 + 16 * i + l, (int64_t)m - 1) * ldp;
#pragma unroll
    for (int i = 0; i < NT; ++i)
        qr[i] = q + min(r0 + 16 * i + l, (int64_t)n - 1) * ldq;
    i32x4 acc[MT][NT] = {};
    // (a lane's k past the end: a zero code on the weight's side is enough)
    const int32_t steps = (k + 63) / 64, each = (steps + W - 1) / W;
    const int32_t u1 = min(steps, (wave + 1) * each);
#pragma unroll(MT *NT > 4 ? 2 : 4)
    for (int32_t u = wave * each; u < u1; ++u) {
        const int32_t c = u * 64 + g * 16, at = min(c, k - 16);
        i32x4 a[MT], b[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            a[i] = *reinterpret_cast<const i32x4 *>(pj[i] + at);
            a[i] = c < k ? a[i] : zero;
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
            b[i] = *reinterpret_cast<const i32x4 *>(qr[i] + at);
#pragma unroll
        for (int h = 0; h < MT; ++h)
#pragma unroll
            for (int i = 0; i < NT; ++i)
                acc[h][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[h], b[i], acc[h][i], 0, 0, 0);
    }
#pragma unroll
    for (int h = 0; h < MT; ++h)
#pragma unroll
        for (int i = 0; i < NT; ++i)
            red[wave][h * NT + i][lane] = acc[h][i];
    __syncthreads();
    for (int x = wave; x < MT * NT; x += W) {
        i32x4 v = red[0][x][lane];
#pragma unroll
        for (int w = 1; w < W; ++w)
            v += red[w][x][lane];
        const int64_t r = r0 + x % NT * 16 + l;
        const int sum[4] = {v[0], v[1], v[2], v[3]};
        if (r < n)
            store_row(sum, s[r], t, relu, j0 + x / NT * 16 + 4 * g, m, y + r * ldy);
    }
}

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;
__device__ const uint4 kZeros = {0, 0, 0, 0};

// A tile of BN rows x BM channels a workgroup, 16 TM channels x 64 rows a wave
// (WM x WN waves).  The channels are the instruction's rows, so that a lane
// holds channels in a row of one output row.  Lines of 64 k of both operands
// come straight into a ring of places in LDS: 16 rows of 64 bytes are a block
// of 1 KB, the 16-byte piece c of row r at place c ^ (r / 2 % 4), so that the
// lanes of a read (16 rows, one piece each) fall on different banks.  The sums are
// whole numbers below 2^31 (k <= 65536), exact in any order.
//
// With 16-bit outputs the channels of a pair of blocks are dealt to the block's
// rows so that a lane holds eight in a row.
//
// 8,192 x 4,096 x 4,096 bfloat16 out at 256 x 256: 126 to 144 us, 1.9 to 2.2 P
// operations a second; the matrix units are busy half the time at the 2.1 GHz that
// the card's power leaves.  (Fragments read a line ahead, between the matrix
// instructions: 145 against 152 us there, but 90 against 84 for 16,384 x 640 x 4,096;
// not kept.)
template <class T, int WM, int WN, int TM>
__global__ __launch_bounds__(WM *WN *kWave) void k_q8_gemm(
    int32_t n, int32_t m, int32_t k, int32_t tiles_m, const int8_t *__restrict__ q, int64_t ldq,
    const float *__restrict__ s, const int8_t *__restrict__ p, int64_t ldp,
    const float *__restrict__ t, bool relu, T *__restrict__ y, int64_t ldy)
{
    constexpr int W = WM * WN, TN = 4, BM = WM * TM * 16, BN = WN * TN * 16;
    constexpr int BLOCKS = (BM + BN) / 16, L = BLOCKS / W, RING = 4;
    static_assert(BLOCKS % W == 0 && TM % 2 == 0, "every wave loads as much");
    __shared__ i32x4 lds0[BLOCKS * kWave], lds1[BLOCKS * kWave], lds2[BLOCKS * kWave],
        lds3[BLOCKS * kWave];

    const int lane = threadIdx.x % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int64_t j0 = (int64_t)(id % tiles_m) * BM, r0 = (int64_t)(id / tiles_m) * BN;

    // what this lane loads of each of its blocks: row lane / 4, place lane % 4
    const int8_t *src[L];
    const int lr = lane / 4, lc = (lane % 4 ^ lr / 2 % 4) * 16;
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int blk = i * W + wave;
        if (blk < BM / 16) {
            const int ch = sizeof(T) == 2 ? blk / 2 * 32 + lr / 4 * 8 + blk % 2 * 4 + lr % 4
                                          : blk * 16 + lr;
            src[i] = p + min(j0 + ch, (int64_t)m - 1) * ldp + lc;
        } else {
            src[i] = q + min(r0 + (blk - BM / 16) * 16 + lr, (int64_t)n - 1) * ldq + lc;
        }
    }
    auto load_one = [&](int32_t line, i32x4 *dst, int i) {
        const void *from = line * 64 + lc < k ? (const void *)(src[i] + line * 64)
                                              : (const void *)&kZeros;
        __builtin_amdgcn_global_load_lds((global_void *)from,
                                         (lds_void *)(&dst[(i * W + wave) * kWave]), 16, 0, 0);
    };
    auto load = [&](int32_t line, i32x4 *dst) {
#pragma unroll
        for (int i = 0; i < L; ++i)
            load_one(line, dst, i);
    };
    // Waits until all but the wave's newest `lines` lines are in LDS and its reads
    // are done, then for the other waves.
    static_assert((RING - 1) * L < 64, "vmcnt holds six bits");
    auto sync = [&](auto lines) {
        constexpr int c = decltype(lines)::value * L;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((c & 15) | 7 << 4 | (c >> 4) << 14);
        asm volatile("s_barrier" ::: "memory");
    };
    const int l = lane % 16, g = lane / 16;
    const int read = l * 4 + (g ^ l / 2 % 4);
    const int wm = wave / WN * TM, wn = BM / 16 + wave % WN * TN;

    i32x4 acc[TM][TN] = {};
    const int32_t lines = (k + 63) / 64;
    // One line.  The place of the line before, which every wave has read at the
    // barrier, is loaded with the line RING - 1 ahead of this one.  (Past the last
    // line zeros are loaded, so that the waits count alike.)
    auto step = [&](int32_t line, const i32x4 *now, i32x4 *free) {
        sync(std::integral_constant<int, RING - 2>());
        i32x4 a[TM], b[TN];
#pragma unroll
        for (int i = 0; i < TN; ++i)
            b[i] = now[(wn + i) * kWave + read];
#pragma unroll
        for (int i = 0; i < TM; ++i)
            a[i] = now[(wm + i) * kWave + read];
        load(line + RING - 1, free);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int h = 0; h < TN; ++h)
                acc[i][h] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], b[h], acc[i][h], 0, 0, 0);
    };
    load(0, lds0);
    load(1, lds1);
    load(2, lds2);
    int32_t line = 0;
    for (; line + 4 <= lines; line += 4) {
        step(line, lds0, lds3);
        step(line + 1, lds1, lds0);
        step(line + 2, lds2, lds1);
        step(line + 3, lds3, lds2);
    }
    if (line < lines)
        step(line, lds0, lds3);
    if (line + 1 < lines)
        step(line + 1, lds1, lds0);
    if (line + 2 < lines)
        step(line + 2, lds2, lds1);
    // (no load may still be under way to LDS when the workgroup's ends)
    __builtin_amdgcn_s_waitcnt(0);

#pragma unroll
    for (int h = 0; h < TN; ++h) {
        const int64_t r = r0 + (wn - BM / 16 + h) * 16 + l;
        if (r >= n)
            continue;
        const float sr = s[r];
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < TM; i += 2) {
                const int sum[8] = {acc[i][h][0], acc[i][h][1], acc[i][h][2], acc[i][h][3],
                                    acc[i + 1][h][0], acc[i + 1][h][1], acc[i + 1][h][2],
                                    acc[i + 1][h][3]};
                store_row(sum, sr, t, relu, j0 + (wm + i) * 16 + g * 8, m, y + r * ldy);
            }
        } else {
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int sum[4] = {acc[i][h][0], acc[i][h][1], acc[i][h][2], acc[i][h][3]};
                store_row(sum, sr, t, relu, j0 + (wm + i) * 16 + g * 4, m, y + r * ldy);
            }
        }
    }
}

// Many rows by a weight of at most 64 LINES of k, 16 MB channels a workgroup:
// bound by writing y.  The weight's codes stay in LDS (in the places of
// k_q8_gemm), and each wave takes 16 rows after another straight from memory, the
// next ones' codes under way while these are multiplied and stored; no barrier
// after the first.  306,250 x 256 x 256 float32 out 80 to 91 us (4.3 to 4.9 TB/s),
// 300,000 x 600 x 256 bfloat16 89 (3.8), 16,384 x 640 x 4,096 74 (1.2 P operations a
// second, of which 27 to store y).
// (Kept to 128 registers, two workgroups a compute unit: 121; stores past the
// caches 93; rows in runs a wave instead of interleaved 97.)
template <class T, int LINES, int MB, int W>
__global__ __launch_bounds__(W *kWave) void k_q8_stream(
    int32_t n, int32_t m, int32_t k, const int8_t *__restrict__ q, int64_t ldq,
    const float *__restrict__ s, const int8_t *__restrict__ p, int64_t ldp,
    const float *__restrict__ t, bool relu, T *__restrict__ y, int64_t ldy)
{
    static_assert(sizeof(T) == 4 || MB % 2 == 0, "pairs of blocks");
    __shared__ i32x4 lds[LINES * MB * kWave];
    __shared__ float lt[16 * MB];
    const int lane = threadIdx.x % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int l = lane % 16, g = lane / 16;
    const int64_t j0 = (int64_t)blockIdx.y * (16 * MB);
    // the channel of row r of block b: with 16-bit outputs a pair's are dealt so
    // that a lane holds eight in a row
    auto channel = [](int b, int r) {
        return sizeof(T) == 2 ? b / 2 * 32 + r / 4 * 8 + b % 2 * 4 + r % 4 : b * 16 + r;
    };
    const int lr = lane / 4, lc = (lane % 4 ^ lr / 2 % 4) * 16;
    for (int i = wave; i < LINES * MB; i += W) {
        const int64_t j = j0 + channel(i % MB, lr);
        const int32_t c = i / MB * 64 + lc;
        const void *from = j < m && c < k ? (const void *)(p + j * ldp + c) : (const void *)&kZeros;
        __builtin_amdgcn_global_load_lds((global_void *)from, (lds_void *)(&lds[i * kWave]), 16, 0,
                                         0);
    }
    for (int i = threadIdx.x; i < 16 * MB; i += W * kWave)
        lt[i] = j0 + i < m ? t[j0 + i] : 0.f;
    __builtin_amdgcn_s_waitcnt(0);   // (the loads to LDS)
    __syncthreads();
    const int read = l * 4 + (g ^ l / 2 % 4);

    struct Rows {
        i32x4 q[LINES];
        float s;
    };
    // (codes past k meet the weight's zeros)
    auto fetch = [&](int64_t r0, Rows &f) {
        const int64_t r = min(r0 + l, (int64_t)n - 1);
        f.s = s[r];
#pragma unroll
        for (int u = 0; u < LINES; ++u)
            f.q[u] = *reinterpret_cast<const i32x4 *>(q + r * ldq + min(u * 64 + g * 16, k - 16));
    };
    const int64_t stride = (int64_t)gridDim.x * W * 16;
    int64_t r0 = ((int64_t)blockIdx.x * W + wave) * 16;
    Rows now, next;
    if (r0 < n)
        fetch(r0, now);
    for (; r0 < n; r0 += stride) {
        fetch(min(r0 + stride, (int64_t)n - 1), next);
        // (the weight's codes are read again for each 16 rows, not kept in registers)
        asm volatile("" ::: "memory");
        i32x4 acc[MB] = {};
#pragma unroll
        for (int u = 0; u < LINES; ++u)
#pragma unroll
            for (int b = 0; b < MB; ++b) {
                acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(lds[(u * MB + b) * kWave + read],
                                                               now.q[u], acc[b], 0, 0, 0);
                if (b % 4 == 3)
                    __builtin_amdgcn_sched_barrier(0);   // (no more reads ahead)
            }
        if (r0 + l < n) {
            T *yr = y + (r0 + l) * ldy + j0;
            // (what the stores need is formed here, not kept through the loop)
            int32_t left = (int32_t)(m - j0);
            int at = g;
            asm volatile("" : "+s"(left), "+v"(at));
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int b = 0; b < MB; b += 2) {
                    const int sum[8] = {acc[b][0], acc[b][1], acc[b][2], acc[b][3],
                                        acc[b + 1][0], acc[b + 1][1], acc[b + 1][2],
                                        acc[b + 1][3]};
                    store_row(sum, now.s, lt, relu, b * 16 + at * 8, left, yr);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
#pragma unroll
                for (int b = 0; b < MB; ++b) {
                    const int sum[4] = {acc[b][0], acc[b][1], acc[b][2], acc[b][3]};
                    store_row(sum, now.s, lt, relu, b * 16 + at * 4, left, yr);
                    if (b % 4 == 3)
                        __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        now = next;
    }
}

// dw over rows [z chunk, (z + 1) chunk) into slice z: TC columns of codes x TJ
// of D a workgroup of 8 waves, 32 rows a step, 64 for the smaller tiles.  The codes are exact in
// bfloat16; s D is split into three bfloat16 by cutting off its low bits,
// which together are exactly its 24 bits, so that the products are exact and
// the sums fp32.
//
// A thread fetches four columns of four rows, a step ahead in
// registers, and leaves them in LDS beside the step before's instructions, as
// the matrix instructions take them: [rows / 8][slot] pieces of 16 bytes, slot
// i T / 4 + q holding column 4 q + i, so that neighbouring lanes write
// neighbouring bytes (two lanes a piece) and a wave's four tiles of D give each
// lane 16 columns in a row of dw to store.
//
// Bound by memory where dw is small, by the matrix instructions where it is not:
// 306,250 x 256 x 256 float32 with ReLU 142 to 169 us and 12 for the slices' sum
// (4.2 to 5.0 TB/s), 16,384 x 1,024 x 4,096 bfloat16 328 to 400 us one after another
// and about 298 between other work, and 17 (1.0 to 1.4 PFLOP/s of three products
// each, by the clock that the card's power leaves; a large library product reaches
// 1.1 to 1.25 here).  Tried on the former, 145 us at the time: tiles of 128 x 128
// 288 us, 128 x 256 217, 256 x 128 213 (each step costs about the same whatever
// the tile); a second set of fetched registers 213 to 813 (spills, or waits that
// the compiler cannot count over branches).  29,125 x 602 x 256: 43 us and 11; its
// 85 slices' stores and 11 steps of 2.4 us, in which operands, splitting and
// products take turns.
constexpr int kGradRows = 32, kGradThreads = 512;
// 32s of rows in a step: a step costs about the same whatever it holds.
constexpr int grad_blocks(int tc, int tj) { return tc * tj <= 16384 ? 2 : 1; }
template <int TILE>
__device__ __forceinline__ int slot_column(int slot)
{
    return slot % (TILE / 4) * 4 + slot / (TILE / 4);
}
// ANY: fewer than four columns, or strides whose offsets of a step's rows pass 32
// bits; element by element.
template <class T, bool RELU, int TC, int TJ, bool ANY>
__global__ __launch_bounds__(kGradThreads) void k_q8_grad(
    int32_t n, int32_t k, int32_t m, int64_t chunk, int32_t splits, int32_t tiles_c,
    int32_t tiles_j, const int8_t *__restrict__ q, int64_t ldq, const float *__restrict__ s,
    const T *__restrict__ dy, int64_t lddy, const T *__restrict__ y, int64_t ldy,
    float *__restrict__ part)
{
    constexpr int WJ = TJ / 64, WC = 8 / WJ, CW = TC / WC, NI = CW / 16;
    constexpr int R = grad_blocks(TC, TJ), ROWS = R * kGradRows;
    // vectors of four columns x four rows of D and of codes, and a thread's
    constexpr int UD = TJ * 2 * R, UC = TC * 2 * R;
    constexpr int ND = UD > kGradThreads ? UD / kGradThreads : 1;
    constexpr int NC = UC > kGradThreads ? UC / kGradThreads : 1;
    constexpr int HD = 2 * kGradThreads / TJ, HC = 2 * kGradThreads / TC;   // octets apart
    static_assert(NI >= 1 && ND <= R && NC <= R, "a place for each beside the products");
    // [buffer](part)[octet][slot][half]
    __shared__ bf16x4 lc[2][4 * R][TC][2], ld[2][3][4 * R][TJ][2];

    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const uint32_t id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int32_t tile = id % (tiles_c * tiles_j), z = id / (tiles_c * tiles_j);
    const int64_t c0 = (int64_t)(tile / tiles_j) * TC, j0 = (int64_t)(tile % tiles_j) * TJ;
    const int64_t rb = z * chunk, re = min((int64_t)n, rb + chunk);

    const int half = tid % 2;
    // (threads with nothing to fetch repeat others' fetches)
    const int qd = tid / 2 % (TJ / 4), od = tid / 2 / (TJ / 4) % (4 * R);
    const int qc = tid / 2 % (TC / 4), oc = tid / 2 / (TC / 4) % (4 * R);
    const bool does_d = UD >= kGradThreads || tid < UD, does_c = UC >= kGradThreads || tid < UC;
    // A vector that would pass the row's end lies against it instead: its columns
    // are formed twice, alike.  Vectors behind it repeat it and are not stored.
    const int64_t last = max(m - 4, 0);
    const int64_t jd = min(j0 + 4 * qd, last), cc = min(c0 + 4 * qc, (int64_t)q8_padded(k) - 4);

    const int rd = od * 8 + half * 4, rc = oc * 8 + half * 4;
    const uint32_t bytes_d = lddy * sizeof(T), bytes_y = ldy * sizeof(T), bytes_c = ldq;
    const uint32_t col_d = jd * sizeof(T), col_c = cc;   // (not with ANY)
    struct Fetched {
        typename Vec<T, 4>::type d[ND][4], y[RELU ? ND : 1][4];
        typename Vec<float, 4>::type s[ND];
        uint32_t c[NC][4];
    } next;
    // The rows r0 .. r0 + ROWS - 1.  Rows past the end repeat the last one with
    // codes of zero: what it adds to its columns is nothing, or the NaN that they
    // hold.
    auto fetch = [&](Fetched &f, int64_t r0) {
        const int rows = (int)min((int64_t)ROWS, re - r0);
        if (rows <= 0)
            return;
        const char *bd = (const char *)(dy + r0 * lddy), *by = (const char *)(y + r0 * ldy);
        const char *bc = (const char *)(q + r0 * ldq), *bs = (const char *)(s + r0);
        if constexpr (ANY) {
#pragma unroll
            for (int x = 0; x < ND; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t r = r0 + min(rd + x * HD * 8 + i, rows - 1);
                    f.s[x][i] = s[r];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t j = min(jd + e, (int64_t)m - 1);
                        f.d[x][i][e] = dy[r * lddy + j];
                        if constexpr (RELU)
                            f.y[x][i][e] = y[r * ldy + j];
                    }
                }
#pragma unroll
            for (int x = 0; x < NC; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = rc + x * HC * 8 + i;
                    f.c[x][i] = r < rows ? *reinterpret_cast<const uint32_t *>(
                                               q + (r0 + r) * ldq + cc)
                                         : 0;
                }
            return;
        }
        typedef typename Vec<T, 4>::type vec;
        if (rows == ROWS) {
            const uint32_t at_d = rd * bytes_d + col_d, at_y = rd * bytes_y + col_d;
            const uint32_t at_c = rc * bytes_c + col_c;
#pragma unroll
            for (int x = 0; x < ND; ++x) {
                f.s[x] = *reinterpret_cast<const typename Vec<float, 4>::type *>(
                    bs + x * HD * 32 + (uint32_t)rd * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint64_t r = x * HD * 8 + i;
                    f.d[x][i] = *reinterpret_cast<const vec *>(bd + r * bytes_d + at_d);
                    if constexpr (RELU)
                        f.y[x][i] = *reinterpret_cast<const vec *>(by + r * bytes_y + at_y);
                }
            }
#pragma unroll
            for (int x = 0; x < NC; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    f.c[x][i] = *reinterpret_cast<const uint32_t *>(
                        bc + (uint64_t)(x * HC * 8 + i) * bytes_c + at_c);
        } else {
#pragma unroll
            for (int x = 0; x < ND; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t r = min(rd + x * HD * 8 + i, rows - 1);
                    f.s[x][i] = *reinterpret_cast<const float *>(bs + r * 4);
                    f.d[x][i] = *reinterpret_cast<const vec *>(bd + (r * bytes_d + col_d));
                    if constexpr (RELU)
                        f.y[x][i] = *reinterpret_cast<const vec *>(by + (r * bytes_y + col_d));
                }
#pragma unroll
            for (int x = 0; x < NC; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = rc + x * HC * 8 + i;
                    const uint32_t h = min(r, rows - 1);
                    f.c[x][i] = *reinterpret_cast<const uint32_t *>(bc + (h * bytes_c + col_c));
                    f.c[x][i] = r < rows ? f.c[x][i] : 0;
                }
        }
    };
    // column i of what was fetched, into buffer b
    auto stash_codes = [&](const Fetched &f, int b, int x, int i) {
        if (!does_c)
            return;
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = (__bf16)(float)(int8_t)(f.c[x][e] >> (8 * i));
        lc[b][oc + x * HC][i * (TC / 4) + qc][half] = v;
    };
    auto stash_d = [&](const Fetched &f, int b, int x, int i) {
        if (!does_d)
            return;
        bf16x4 v[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float D = (float)f.d[x][e][i];
            if constexpr (RELU)
                if (!((float)f.y[x][e][i] > 0.f))
                    D = 0.f;
            D *= f.s[x][e];
#pragma unroll
            for (int h = 0; h < 3; ++h) {
                const uint32_t top = __float_as_uint(D) & 0xffff0000u;
                v[h][e] = __builtin_bit_cast(__bf16, (uint16_t)(top >> 16));
                D -= __uint_as_float(top);
            }
        }
#pragma unroll
        for (int h = 0; h < 3; ++h)
            ld[b][h][od + x * HD][i * (TJ / 4) + qd][half] = v[h];
    };
    // the parts of a step's stash: a column of each of the thread's vectors
    constexpr int PARTS = 4 * (ND + NC);
    auto stash = [&](const Fetched &f, int b, int part) {
        const int i = part % 4, x = part / 4;
        if (x < ND)
            stash_d(f, b, x, i);
        else
            stash_codes(f, b, x - ND, i);
    };

    f32x4 acc[NI][4] = {};
    const int l = lane % 16, g = lane / 16;
    const int wj = wave % WJ, wc = wave / WJ;
    auto step = [&](int b, Fetched &next, int64_t further) {
        lds_barrier();
        bf16x8 c[NI];
        auto codes = [&](int sub) {
#pragma unroll
            for (int o = 0; o < NI; ++o)
                c[o] = *reinterpret_cast<const bf16x8 *>(
                    &lc[b][4 * sub + g][wc * CW + o * 16 + l][0]);
        };
        // (a fragment is read beside the instructions that take the one before)
        auto frag = [&](int slot) {
            return *reinterpret_cast<const bf16x8 *>(
                &ld[b][2 - slot % 3][slot / 12 * 4 + g][slot % 12 / 3 * (TJ / 4) + wj * 16 + l][0]);
        };
        codes(0);
        bf16x8 a = frag(0), ahead;
#pragma unroll
        for (int slot = 0; slot < 12 * R; ++slot) {
            if (slot > 0 && slot % 12 == 0)
                codes(slot / 12);
            if (slot < 12 * R - 1)
                ahead = frag(slot + 1);
#pragma unroll
            for (int o = 0; o < NI; ++o)
                acc[o][slot % 12 / 3] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    a, c[o], acc[o][slot % 12 / 3], 0, 0, 0);
            // the next step's operands, beside the last instructions
            if (slot >= 12 * R - PARTS)
                stash(next, b ^ 1, slot - (12 * R - PARTS));
            a = ahead;
            __builtin_amdgcn_sched_barrier(0);
        }
        fetch(next, further);
    };
    fetch(next, rb);
#pragma unroll
    for (int part = 0; part < PARTS; ++part)
        stash(next, 0, part);
    fetch(next, rb + ROWS);
    int b = 0;
    for (int64_t r0 = rb; r0 < re; r0 += ROWS, b ^= 1)
        step(b, next, r0 + 2 * ROWS);
    if (splits > 1) {
        // as the lanes hold them
        f32x4 *out = (f32x4 *)part + ((int64_t)z * (tiles_c * tiles_j) + tile) * (TC * TJ / 4) +
                     wave * (NI * 4 * kWave) + lane;
#pragma unroll
        for (int o = 0; o < NI; ++o)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                out[(o * 4 + i) * kWave] = acc[o][i];
        return;
    }
#pragma unroll
    for (int o = 0; o < NI; ++o) {
        const int64_t c = c0 + slot_column<TC>(wc * CW + o * 16 + l);
        if (c >= k)
            continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t j = j0 + 4 * (wj * 16 + g * 4 + e);
            float *p = part + c * m + min(j, last);
            if (j >= m)
                continue;
            if (m >= 4) {
                typename Vec<float, 4>::type v;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[i] = acc[o][i][e];
                *reinterpret_cast<typename Vec<float, 4>::type *>(p) = v;
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (i < m)
                        p[i] = acc[o][i][e];
            }
        }
    }
}

// Few rows: 64 columns of codes x 64 of D a workgroup, its 8 waves a run of the
// rows each, straight from memory into the matrix instructions' operands (four
// columns a lane and load, as above); the waves' sums are added in their order
// through LDS, and dw is written at once.
template <class T, bool RELU>
__global__ __launch_bounds__(kGradThreads) void k_q8_grad_few(
    int32_t n, int32_t k, int32_t m, const int8_t *__restrict__ q, int64_t ldq,
    const float *__restrict__ s, const T *__restrict__ dy, int64_t lddy, const T *__restrict__ y,
    int64_t ldy, float *__restrict__ dw)
{
    constexpr int W = kGradThreads / kWave;
    typedef typename Vec<T, 4>::type vec;
    __shared__ f32x4 red[W][4][4][kWave];
    const int lane = threadIdx.x % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int l = lane % 16, g = lane / 16;
    const int64_t c0 = (int64_t)blockIdx.x * 64, j0 = (int64_t)blockIdx.y * 64;
    const int64_t last = max(m - 4, 0);
    const int64_t jd = min(j0 + 4 * l, last), cc = min(c0 + 4 * l, (int64_t)q8_padded(k) - 4);
    const int64_t each = ((int64_t)n + W * kGradRows - 1) / (W * kGradRows) * kGradRows;
    const int64_t rb = wave * each, re = min((int64_t)n, rb + each);
    f32x4 acc[4][4] = {};
    for (int64_t r0 = rb; r0 < re; r0 += kGradRows) {
        vec d[8], h[RELU ? 8 : 1];
        uint32_t c[8];
        float sr[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // (rows past the end repeat the last one, with codes of zero)
            const bool there = r0 + g * 8 + e < re;
            const int64_t r = min(r0 + g * 8 + e, re - 1);
            sr[e] = s[r];
            c[e] = there ? *reinterpret_cast<const uint32_t *>(q + r * ldq + cc) : 0;
            if (m >= 4) {
                d[e] = *reinterpret_cast<const vec *>(dy + r * lddy + jd);
                if constexpr (RELU)
                    h[e] = *reinterpret_cast<const vec *>(y + r * ldy + jd);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    d[e][i] = dy[r * lddy + min(i, m - 1)];
                    if constexpr (RELU)
                        h[e][i] = y[r * ldy + min(i, m - 1)];
                }
            }
        }
        bf16x8 cf[4];
#pragma unroll
        for (int o = 0; o < 4; ++o)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                cf[o][e] = (__bf16)(float)(int8_t)(c[e] >> (8 * o));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bf16x8 a[3];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float D = (float)d[e][i];
                if constexpr (RELU)
                    if (!((float)h[e][i] > 0.f))
                        D = 0.f;
                D *= sr[e];
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    const uint32_t top = __float_as_uint(D) & 0xffff0000u;
                    a[p][e] = __builtin_bit_cast(__bf16, (uint16_t)(top >> 16));
                    D -= __uint_as_float(top);
                }
            }
#pragma unroll
            for (int p = 2; p >= 0; --p)
#pragma unroll
                for (int o = 0; o < 4; ++o)
                    acc[o][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[p], cf[o], acc[o][i], 0,
                                                                        0, 0);
        }
    }
#pragma unroll
    for (int o = 0; o < 4; ++o)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            red[wave][o][i][lane] = acc[o][i];
    __syncthreads();
    if (wave >= 4)
        return;
    f32x4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = red[0][wave][i][lane];
#pragma unroll
        for (int w = 1; w < W; ++w)
            v[i] += red[w][wave][i][lane];
    }
    const int64_t c = c0 + 4 * l + wave;
    if (c >= k)
        return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t j = j0 + 4 * (g * 4 + e);
        float *p = dw + c * m + min(j, last);
        if (j >= m)
            continue;
        if (m >= 4) {
            const typename Vec<float, 4>::type r = {v[0][e], v[1][e], v[2][e], v[3][e]};
            *reinterpret_cast<typename Vec<float, 4>::type *>(p) = r;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < m)
                    p[i] = v[i][e];
        }
    }
}

// dw = the sum of the slices, each tile's vectors as k_q8_grad's lanes hold them.
// Many slices (FEW false): 64 vectors a workgroup, whose 16 waves sum a run of
// slices each, in their order, and then the waves' sums in theirs.  Few: 256
// vectors, 64 a wave, which together are whole runs of dw's rows to store.
constexpr int kSumWaves = 16, kSumFew = 32;
template <int TC, int TJ, bool FEW>
__global__ __launch_bounds__(FEW ? 4 * kWave : kSumWaves *kWave) void k_q8_grad_sum(
    const float *__restrict__ part, int32_t splits, int32_t k, int32_t m, int32_t tiles_j,
    int64_t slice, float *__restrict__ dw)
{
    constexpr int WJ = TJ / 64, WC = 8 / WJ, CW = TC / WC, NI = CW / 16, EACH = 8 * NI;
    constexpr int WAVES = FEW ? 4 : kSumWaves;
    __shared__ f32x4 red[WAVES][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int block = FEW ? blockIdx.x : blockIdx.x / 4;
    const int i = FEW ? wave : blockIdx.x % 4;   // column of four
    const int32_t each = FEW ? splits : (splits + WAVES - 1) / WAVES;
    const int32_t z0 = FEW ? 0 : wave * each, z1 = min(splits, z0 + each);
    const f32x4 *src = (const f32x4 *)part + ((int64_t)block * 4 + i) * kWave + lane;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int32_t z = z0; z < z1; ++z)
        v += src[z * slice];
    red[wave][lane] = v;
    __syncthreads();
    // what the lane holds there
    const int tile = block / EACH, of = block % EACH / NI, o = block % NI;
    const int64_t c = (int64_t)(tile / tiles_j) * TC +
                      slot_column<TC>(of / WJ * CW + o * 16 + lane % 16);
    if (c >= k)
        return;
    const int64_t last = max(m - 4, 0);
    const int64_t j0 = (int64_t)(tile % tiles_j) * TJ + 4 * (of % WJ * 16 + lane / 16 * 4);
    if constexpr (FEW) {
        // row `wave` of the lane's four
        const int64_t j = j0 + 4 * wave;
        if (j >= m)
            return;
        typename Vec<float, 4>::type r;
#pragma unroll
        for (int h = 0; h < 4; ++h)
            r[h] = red[h][lane][wave];
        float *p = dw + c * m + min(j, last);
        if (m >= 4) {
            *reinterpret_cast<typename Vec<float, 4>::type *>(p) = r;
        } else {
#pragma unroll
            for (int h = 0; h < 3; ++h)
                if (h < m)
                    p[h] = r[h];
        }
    } else {
        if (wave > 0)
            return;
#pragma unroll
        for (int w = 1; w < WAVES; ++w)
            v += red[w][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (j0 + 4 * e < m && i < m)
                dw[c * m + min(j0 + 4 * e, last) + i] = v[e];
    }
}

template <class T>
struct Tag {
    typedef T type;
};

template <class F>
hipError_t with_type(int32_t type, F f)
{
    if (type == kF32)
        return f(Tag<float>{});
    if (type == kBF16)
        return f(Tag<__bf16>{});
    return f(Tag<_Float16>{});
}

// Launches over rows [r0, r0 + n), at most kTurn at a time: a grid's threads are
// counted in 32 bits.
constexpr int32_t kTurn = 1 << 21;
template <class F>
hipError_t in_turns(int32_t n, F f)
{
    for (int64_t r0 = 0; r0 < n; r0 += kTurn)
        if (hipError_t e = f((int64_t)r0, (int32_t)std::min<int64_t>(kTurn, n - r0)))
            return e;
    return hipSuccess;
}

RowList from(RowList l, int64_t r0)
{
    if (l.p)
        l.p = (const char *)l.p + r0 * (l.wide ? 8 : 4);
    return l;
}

template <class T, int GL, int Q, int WAVES>
hipError_t quantize(int32_t n, int32_t d, const T *x, int64_t ldx, RowList src, int64_t n_x,
                    int8_t *codes, int64_t ldq, float *scales, RowList dst, hipStream_t s)
{
    const int rows = WAVES == 1 ? kThreads / GL : 1;
    const uint32_t blocks = (uint32_t)(((int64_t)n + rows - 1) / rows);
    k_quantize_rows<T, GL, Q, WAVES>
        <<<blocks, WAVES == 1 ? kThreads : WAVES * kWave, 0, s>>>(n, d, x, ldx, src, n_x, codes,
                                                                  ldq, scales, dst);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(int32_t type, int32_t n, int32_t d, const void *x, int64_t ldx,
                                RowList src, int64_t n_x, int8_t *codes, int64_t ldq,
                                float *scales, RowList dst, hipStream_t s)
{
    return in_turns(n, [&](int64_t r0, int32_t n) { return with_type(type, [&](auto tag) {
        typedef typename decltype(tag)::type T;
        const int vectors = (q8_padded(d) + kVecOf<T> - 1) / kVecOf<T>;
        auto run = [&](auto f) {
            return f(n, d, (const T *)x + (src.p ? 0 : r0 * ldx), ldx, from(src, r0),
                     src.p ? n_x : n, codes + (dst.p ? 0 : r0 * ldq), ldq,
                     scales + (dst.p ? 0 : r0), from(dst, r0), s);
        };
        if (vectors <= 8)
            return run(quantize<T, 4, 2, 1>);
        if (vectors <= 16)
            return run(quantize<T, 4, 4, 1>);
        if (vectors <= 32)
            return run(quantize<T, 8, 4, 1>);
        if (vectors <= 64)
            return run(quantize<T, 16, 4, 1>);
        if (vectors <= 128)
            return run(quantize<T, 32, 4, 1>);
        if (vectors <= 256)
            return run(quantize<T, 64, 4, 1>);
        if (vectors <= 1024)
            return run(quantize<T, 64, 4, 4>);
        if (vectors <= 4096)
            return run(quantize<T, 64, 4, 16>);
        return run(quantize<T, 64, 16, 16>);
    }); });
}

hipError_t launch_quantize_columns(int32_t type, int32_t rows, int32_t cols, const void *w,
                                   int64_t ldw, int8_t *codes, int64_t ldq, float *scales,
                                   hipStream_t s)
{
    return with_type(type, [&](auto tag) {
        typedef typename decltype(tag)::type T;
        auto run = [&](auto c, auto p) {
            constexpr int C = decltype(c)::value, P = decltype(p)::value;
            k_quantize_columns<T, C, P><<<(cols + C - 1) / C, kColThreads, 0, s>>>(
                rows, cols, (const T *)w, ldw, codes, ldq, scales);
            return hipGetLastError();
        };
        // few columns: four a workgroup, so that more of them share the rows
        if (cols <= 1024 && rows <= 4096)
            return run(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
        if (rows <= 1024)
            return run(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
        if (rows <= 4096)
            return run(std::integral_constant<int, 16>{}, std::integral_constant<int, 4>{});
        return run(std::integral_constant<int, 16>{}, std::integral_constant<int, 0>{});
    });
}

hipError_t launch_dequantize_rows(int32_t type, int32_t n, int32_t d, const int8_t *codes,
                                  int64_t ldq, const float *scales, RowList src, int64_t n_x,
                                  void *y, int64_t ldy, hipStream_t s)
{
    return in_turns(n, [&](int64_t r0, int32_t n) { return with_type(type, [&](auto tag) {
        typedef typename decltype(tag)::type T;
        const int vectors = (d + kVecOf<T> - 1) / kVecOf<T>;
        auto run = [&](auto gl) {
            constexpr int GL = decltype(gl)::value;
            const int rows = kThreads / GL;
            k_dequantize_rows<T, GL, 4>
                <<<(uint32_t)(((int64_t)n + rows - 1) / rows), kThreads, 0, s>>>(
                    n, d, codes + (src.p ? 0 : r0 * ldq), ldq, scales + (src.p ? 0 : r0),
                    from(src, r0), src.p ? n_x : n, (T *)y + r0 * ldy, ldy);
            return hipGetLastError();
        };
        // (Fewer rows, 65,536 x 101 float32: 10.3 us against 9.2.  16-bit rows that
        // leave more than half of their last 16 columns empty: 304,051 x 33 17.8
        // against 15.4, 17 13.0 against 12.2.)
        if (n >= 131072 && ldy == d && d % kVecOf<T> && d <= 256 && (uintptr_t)y % 16 == 0 &&
            (sizeof(T) == 4 || (d - 1) % 16 >= 8)) {
            // (a multiple of 8 rows is one of whole vectors, of either size)
            const int R = std::min(kFlatBytes / q8_padded(d), 256) / 8 * 8;
            k_dequantize_flat<T><<<(n + R - 1) / R, kThreads, 0, s>>>(
                n, d, R, codes + (src.p ? 0 : r0 * ldq), ldq, scales + (src.p ? 0 : r0),
                from(src, r0), src.p ? n_x : n, (T *)y + r0 * ldy);
            return hipGetLastError();
        }
        if (vectors <= 16)
            return run(std::integral_constant<int, 4>{});
        if (vectors <= 32)
            return run(std::integral_constant<int, 8>{});
        if (vectors <= 64)
            return run(std::integral_constant<int, 16>{});
        if (vectors <= 128)
            return run(std::integral_constant<int, 32>{});
        return run(std::integral_constant<int, 64>{});
    }); });
}

hipError_t launch_q8_aggregate(const SpmmBlock *blocks, int32_t n_blocks, int32_t n_long,
                               const int32_t *rowptr, const int32_t *col, const float *val,
                               const int8_t *codes, int64_t ldq, const float *scales, int32_t d,
                               float *out, int64_t ldo, hipStream_t s)
{
    auto run = [&](auto gl) {
        constexpr int GL = decltype(gl)::value;
        if (n_long > 0)
            k_q8_aggregate_long<GL><<<n_long, kSpmmThreads, 0, s>>>(blocks, col, val, codes, ldq,
                                                                   scales, d, out, ldo);
        if (hipError_t e = hipGetLastError())
            return e;
        if (n_blocks > n_long)
            k_q8_aggregate<GL><<<n_blocks - n_long, 8 * GL, 0, s>>>(
                blocks + n_long, rowptr, col, val, codes, ldq, scales, d, out, ldo);
        return hipGetLastError();
    };
    const int32_t pieces = (d + 15) / 16;
    return pieces <= 8    ? run(std::integral_constant<int, 8>{})
           : pieces <= 16 ? run(std::integral_constant<int, 16>{})
           : pieces <= 32 ? run(std::integral_constant<int, 32>{})
                          : run(std::integral_constant<int, 64>{});
}

hipError_t launch_q8_product(int32_t type, int32_t n, int32_t m, int32_t k, const int8_t *q,
                             int64_t ldq, const float *s, const int8_t *p, int64_t ldp,
                             const float *t, bool relu, void *y, int64_t ldy, hipStream_t st)
{
    return in_turns(n, [&](int64_t r0, int32_t n) { return with_type(type, [&](auto tag) {
        typedef typename decltype(tag)::type T;
        // (the turn's rows)
        const int8_t *const qt = q + r0 * ldq;
        const float *const sr = s + r0;
        T *const out = (T *)y + r0 * ldy;
        auto few = [&](auto mt, auto nt) {
            constexpr int MT = decltype(mt)::value, NT = decltype(nt)::value;
            const dim3 grid((m + 16 * MT - 1) / (16 * MT), (n + 16 * NT - 1) / (16 * NT));
            k_q8_few<T, MT, NT, 8><<<grid, 8 * kWave, 0, st>>>(n, m, k, qt, ldq, sr, p, ldp, t,
                                                              relu, out, ldy);
            return hipGetLastError();
        };
        typedef std::integral_constant<int, 1> i1;
        typedef std::integral_constant<int, 2> i2;
        typedef std::integral_constant<int, 4> i4;
        typedef std::integral_constant<int, 6> i6;
        typedef std::integral_constant<int, 8> i8;
        typedef std::integral_constant<int, 10> i10;
        typedef std::integral_constant<int, 12> i12;
        typedef std::integral_constant<int, 16> i16;
        if (n <= 16)
            return few(i1{}, i1{});
        if (n <= 32)
            return few(i1{}, i2{});
        if (n <= 64)
            return few(i1{}, i4{});
        auto gemm = [&](auto wm, auto wn, auto tm) {
            constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value;
            constexpr int TM = decltype(tm)::value, BM = WM * TM * 16, BN = WN * 64;
            const int32_t nm = (m + BM - 1) / BM, nn = (n + BN - 1) / BN;
            k_q8_gemm<T, WM, WN, TM><<<(uint32_t)nm * nn, WM * WN * kWave, 0, st>>>(
                n, m, k, nm, qt, ldq, sr, p, ldp, t, relu, out, ldy);
            return hipGetLastError();
        };
        // The workgroups that the compute units hold at once; where they are no
        // multiple of the groups of channels, more of them with fewer rows each, if
        // there are rows to share (us, once / up to four times: 8,192 x 640 x 20,000
        // bfloat16 235 / 180, 4,096 x 300 x 40,000 145 / 111; 300 x 600 x 20,000 15.0
        // / 17.5, hence the line).
        auto stream = [&](auto lines, auto mb) {
            constexpr int LINES = decltype(lines)::value, MB = decltype(mb)::value;
            constexpr int W = 8;
            const int32_t nm = (m + 16 * MB - 1) / (16 * MB), blocks = (n + 16 * W - 1) / (16 * W);
            int32_t most = LINES > 4 ? 256 : 512;
            while (LINES > 4 && blocks >= 8 && most < 1024 && most / nm * nm < most / 5 * 4)
                most *= 2;
            const dim3 grid(std::max(1, std::min(blocks, most / nm)), nm);
            k_q8_stream<T, LINES, MB, W><<<grid, W * kWave, 0, st>>>(n, m, k, qt, ldq, sr, p, ldp,
                                                                    t, relu, out, ldy);
            return hipGetLastError();
        };
        // The most channels a workgroup that leave every compute unit one (us, 256
        // channels of 256 k, float32, with 256 / 64 channels: 2,048 rows 8.6 / 4.1,
        // 8,192 rows 9.8 / 5.4; of 602 k, with 128 / 64: 8,192 rows 9.2 / 7.3, 29,125
        // rows 18.1 / 21.0; with 256 there, all of LDS, 23.4).  Against tiles through
        // the ring: 29,125 x 256 x 256 float32 11 / 17, 306,250 rows 89 / 140 (4.4
        // TB/s), 300,000 x 600 x 256 bfloat16 89 / 131, 16,384 x 640 x 4,096 74 / 89,
        // 100,000 x 602 x 41 float32 23 / 41, 4,096 x 512 x 4,096 bfloat16 21 / 21.
        auto stream_lines = [&](auto lines) {
            const int64_t blocks = (n + 127) / 128;
            if constexpr (decltype(lines)::value <= 4)
                if (m > 128 && blocks * ((m + 255) / 256) >= 256)
                    return stream(lines, i16{});
            return m > 64 && blocks * ((m + 127) / 128) >= 256 ? stream(lines, i8{})
                                                               : stream(lines, i4{});
        };
        if (k <= 640)
            return k <= 128   ? stream_lines(i2{})
                   : k <= 256 ? stream_lines(i4{})
                   : k <= 384 ? stream_lines(i6{})
                   : k <= 512 ? stream_lines(i8{})
                              : stream_lines(i10{});
        // Workgroups of a tile.  The largest tile that gives every compute unit one
        // reads operands the fewest times (us at 256 x 128 / 128 x 128: 2,048 x 4,096
        // x 4,096 49 / 57); up to 768 k the weight still fits into LDS (100,000 x 768
        // x 256 float32 54 against 65, 16,384 x 768 x 4,096 bfloat16 81 / 95, but
        // 8,192 x 768 x 768 15.9 / 13.4; of 1,024 k 0.96 to 1.17 times as fast).  Where
        // tiles are few the waves share k (1,000 x 2,000 x 300 10.9 / 17.3, 512 x 4,096
        // x 4,096, 512 workgroups, 36 / 21), and no tile is wider than 64 or 128 channels
        // that are all (40,000 x 4,096 x 47 bfloat16 60 / 76, 100,000 x 1,000 x 128
        // float32 65 / 71).
        auto tiles = [&](int bm, int bn) {
            return (int64_t)((m + bm - 1) / bm) * ((n + bn - 1) / bn);
        };
        if (k <= 768 && tiles(256, 256) >= 256)
            return stream_lines(i12{});
        if (m > 128 && tiles(256, 256) >= 256)
            return gemm(i2{}, i4{}, i8{});   // 256 x 256
        if (tiles(64, 64) <= 256)
            return few(i4{}, i4{});
        if (m > 128 && tiles(256, 128) >= 192)
            return gemm(i4{}, i2{}, i4{});   // 256 channels x 128 rows
        if (m > 64)
            return gemm(i4{}, i2{}, i2{});   // 128 x 128
        return gemm(i2{}, i2{}, i2{});       // 64 channels x 128 rows
    }); });
}

namespace {

// Tile sides of the weight gradient: the smallest that hold the matrix, up to
// 256.
int grad_tile_c(int32_t k) { return k > 128 ? 256 : 128; }
int grad_tile_j(int32_t m) { return m > 128 ? 256 : m > 64 ? 128 : 64; }

int64_t grad_tiles(int32_t k, int32_t m, int tc, int tj)
{
    return (int64_t)((k + tc - 1) / tc) * ((m + tj - 1) / tj);
}

// Few rows go without slices (k_q8_grad_few), one workgroup for 64 x 64 of dw
// (us with slices / without: 500 x 64 x 16 float32 9.5 / 7.2, 20 x 1,000 x 1,000 14 /
// 6.1, 500 x 256 x 256 15.4 / 7.7, 1,000 x 1,024 x 1,024 bfloat16 27 / 15, 2,000 rows
// 35 / 25; but 1,000 x 256 x 256 15.7 / 16.7, 2,000 x 602 x 256 20 / 30: few tiles
// of more rows; 1 x 2,000 x 2,000 16 / 19, 1,000 x 4,096 x 4,096 98 / 199: many tiles).
bool grad_few(int32_t n, int32_t k, int32_t m)
{
    const int64_t tiles = (int64_t)((k + 63) / 64) * ((m + 63) / 64);
    return tiles <= 512 && (n <= 512 || (n <= 2048 && tiles >= 64));
}

// Slices of the rows: at most one workgroup a compute unit, and fewer where the
// slices' sums would cost more (written and read once each at about 4.5 TB/s,
// floats of a slice) than the steps that they save (about 2 us each).
int32_t grad_splits(int32_t n, int64_t tiles, int rows, int64_t floats)
{
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(256 / tiles, (int64_t)n / (2 * kGradRows)));
    const double slice = floats * 8 / 4.5e6, blocks = (double)n / rows;
    int64_t best = 1;
    double least = 2.0 * std::ceil(blocks);
    auto consider = [&](int64_t z) {
        const double us = 2.0 * std::ceil(blocks / z) + 4.0 + z * slice;
        if (z > 1 && us < least)
            best = z, least = us;
    };
    // the fewest slices of each number of steps about where the two costs meet
    const double steps = std::ceil(std::sqrt(blocks * slice / 2));
    for (int i = -2; i <= 2; ++i)
        consider(std::min<int64_t>(most,
                                   (int64_t)std::ceil(blocks / std::max(1.0, steps + i))));
    consider(most);
    return (int32_t)best;
}

template <class T, int TC, int TJ, bool ANY>
hipError_t weight_grad(int32_t n, int32_t k, int32_t m, const int8_t *q, int64_t ldq,
                       const float *s, const T *dy, int64_t lddy, const T *y, int64_t ldy,
                       float *part, float *dw, hipStream_t st)
{
    const int32_t nc = (k + TC - 1) / TC, nj = (m + TJ - 1) / TJ;
    const int64_t tiles = (int64_t)nc * nj;
    constexpr int rows = grad_blocks(TC, TJ) * kGradRows;
    const int32_t splits = grad_splits(n, tiles, rows, tiles * TC * TJ);
    int64_t chunk = ((int64_t)n + splits - 1) / splits;
    chunk = (chunk + rows - 1) / rows * rows;
    const auto kernel = y ? k_q8_grad<T, true, TC, TJ, ANY> : k_q8_grad<T, false, TC, TJ, ANY>;
    kernel<<<(uint32_t)(tiles * splits), kGradThreads, 0, st>>>(
        n, k, m, chunk, splits, nc, nj, q, ldq, s, dy, lddy, y, ldy, splits > 1 ? part : dw);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits <= 1)
        return e;
    const int64_t slice = tiles * (TC * TJ / 4);
    if (splits < kSumFew)
        k_q8_grad_sum<TC, TJ, true><<<(uint32_t)(slice / (4 * kWave)), 4 * kWave, 0, st>>>(
            part, splits, k, m, nj, slice, dw);
    else
        k_q8_grad_sum<TC, TJ, false><<<(uint32_t)(slice / kWave), kSumWaves * kWave, 0, st>>>(
            part, splits, k, m, nj, slice, dw);
    return hipGetLastError();
}

}  // namespace

size_t q8_grad_floats(int32_t n, int32_t k, int32_t m)
{
    if (grad_few(n, k, m))
        return 0;
    // with the call's tiles, or the small ones that it takes where strides are
    // too large for them
    size_t most = 0;
    const int sides[2][2] = {{grad_tile_c(k), grad_tile_j(m)}, {128, 64}};
    for (const auto &t : sides) {
        const int64_t tiles = grad_tiles(k, m, t[0], t[1]);
        const int64_t splits = grad_splits(n, tiles, grad_blocks(t[0], t[1]) * kGradRows,
                                           tiles * t[0] * t[1]);
        if (splits > 1)
            most = std::max<size_t>(most, (size_t)(splits * tiles) * t[0] * t[1]);
    }
    return most;
}

int32_t q8_grad_slices(int32_t n, int32_t k, int32_t m)
{
    if (grad_few(n, k, m))
        return 1;
    const int tc = m < 4 ? 128 : grad_tile_c(k), tj = grad_tile_j(m);
    const int64_t tiles = grad_tiles(k, m, tc, tj);
    return grad_splits(n, tiles, grad_blocks(tc, tj) * kGradRows, tiles * tc * tj);
}

hipError_t launch_q8_weight_grad(int32_t type, int32_t n, int32_t k, int32_t m, const int8_t *q,
                                 int64_t ldq, const float *s, const void *dy, int64_t lddy,
                                 const void *y, int64_t ldy, float *part, float *dw,
                                 hipStream_t st)
{
    return with_type(type, [&](auto tag) {
        typedef typename decltype(tag)::type T;
        auto run = [&](auto f) {
            return f(n, k, m, q, ldq, s, (const T *)dy, lddy, (const T *)y, ldy, part, dw, st);
        };
        if (grad_few(n, k, m)) {
            const auto kernel = y ? k_q8_grad_few<T, true> : k_q8_grad_few<T, false>;
            kernel<<<dim3((k + 63) / 64, (m + 63) / 64), kGradThreads, 0, st>>>(
                n, k, m, q, ldq, s, (const T *)dy, lddy, (const T *)y, ldy, dw);
            return hipGetLastError();
        }
        const int64_t pitch = std::max<int64_t>(std::max(lddy, y ? ldy : 0) * sizeof(T), ldq);
        const int tc = grad_tile_c(k), tj = grad_tile_j(m);
        if (m < 4 || (pitch + 65536 * 4) * (2 * kGradRows) > UINT32_MAX)
            return run(weight_grad<T, 128, 64, true>);
        if (tc == 256)
            return tj == 256   ? run(weight_grad<T, 256, 256, false>)
                   : tj == 128 ? run(weight_grad<T, 256, 128, false>)
                               : run(weight_grad<T, 256, 64, false>);
        return tj == 256   ? run(weight_grad<T, 128, 256, false>)
               : tj == 128 ? run(weight_grad<T, 128, 128, false>)
                           : run(weight_grad<T, 128, 64, false>);
    });
}

}  // namespace digest
