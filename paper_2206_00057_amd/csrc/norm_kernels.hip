// gfx950 kernels of the layer norm (forward, backward).
//
// A row of up to 16,384 elements is held in the registers of GL lanes
// (GL <= 64, rows of up to 1,024) or of the WAVES waves of one workgroup, E
// elements a lane in 16-byte vectors, so that x is read once: the mean, then
// the centred squares (two sums over registers, no cancellation), then the
// outputs.  Bound by memory: 306,250 x 256 float32 with ReLU forward 122 us
// (5.2 TB/s; a large copy here runs at 5.1), backward 229 us (5.5 TB/s),
// 16,384 x 4,096 bfloat16 backward 85 us (4.8 TB/s).  Sums are fp32 (over the
// workgroups 64 bits), in a fixed order.  Rows may start at any element: global
// loads and stores take 16-byte vectors at element alignment.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device.h"
#include "train_kernels.h"

namespace digest {
namespace {

constexpr int kThreads = 256;

template <class T>
constexpr int kVecOf = 16 / (int)sizeof(T);

// A vector of T, aligned to its elements only.
template <class T>
struct VecOf {
    typedef T type __attribute__((ext_vector_type(kVecOf<T>), aligned(sizeof(T))));
};

// How the elements behind a row's last whole vector are held: there are none,
// one a lane by the row's first lanes (one more element each), or by the lane
// whose vector they begin, element by element (rows of too few lanes).
enum Rest { kNone, kLanes, kVector };

// The columns that lane l of L lanes holds: vector q starts at (q L + l) V.
template <class T, int E, Rest REST>
struct Columns {
    static constexpr int V = kVecOf<T>, N = E + (REST == kLanes);
    static_assert(E % V == 0, "whole vectors");
    int d, l, L;
    __device__ __forceinline__ int operator()(int e) const
    {
        return REST == kLanes && e == E ? d / V * V + l : ((e / V) * L + l) * V + e % V;
    }
    // element e is one of the row's
    __device__ __forceinline__ bool in(int e) const
    {
        if (REST == kVector)
            return (*this)(e) < d;
        return REST == kLanes && e == E ? l < d % V : (*this)(e / V * V) + V <= d;
    }
    // f[e] = p ? p[column] : dflt, zero past the row's end
    __device__ __forceinline__ void read(const float *__restrict__ p, float dflt,
                                         float (&f)[N]) const
    {
#pragma unroll
        for (int q = 0; q < E / V; ++q) {
            const int c = (*this)(q * V);
            if (c + V <= d) {
#pragma unroll
                for (int j = 0; j < V; j += 4) {
                    typename VecOf<float>::type v = {dflt, dflt, dflt, dflt};
                    if (p)
                        v = *reinterpret_cast<const typename VecOf<float>::type *>(p + c + j);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        f[q * V + j + i] = v[i];
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    f[q * V + j] = REST == kVector && c + j < d ? (p ? p[c + j] : dflt) : 0.f;
            }
        }
        if constexpr (REST == kLanes)
            f[E] = in(E) ? (p ? p[(*this)(E)] : dflt) : 0.f;
    }
};

// A row's elements as its lane holds them; zero past the row's end, and not
// stored there.
template <class T, int E, Rest REST>
struct Row {
    static constexpr int V = kVecOf<T>, Q = E / V;
    typename VecOf<T>::type v[Q];
    T rest;

    __device__ __forceinline__ void load(const T *p, const Columns<T, E, REST> &at)
    {
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int c = at(q * V);
            if (c + V <= at.d) {
                v[q] = *reinterpret_cast<const typename VecOf<T>::type *>(p + c);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    v[q][j] = REST == kVector && c + j < at.d ? p[c + j] : (T)0.f;
            }
        }
        if constexpr (REST == kLanes)
            rest = at.in(E) ? p[at(E)] : (T)0.f;
    }
    __device__ __forceinline__ float operator[](int e) const
    {
        return (float)(e < E ? v[e / V][e % V] : rest);
    }
    __device__ __forceinline__ void set(int e, float x)
    {
        if (e < E)
            v[e / V][e % V] = (T)x;
        else
            rest = (T)x;
    }
    __device__ __forceinline__ void store(T *p, const Columns<T, E, REST> &at) const
    {
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int c = at(q * V);
            if (c + V <= at.d) {
                *reinterpret_cast<typename VecOf<T>::type *>(p + c) = v[q];
            } else if constexpr (REST == kVector) {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (c + j < at.d)
                        p[c + j] = v[q][j];
            }
        }
        if constexpr (REST == kLanes)
            if (at.in(E))
                p[at(E)] = rest;
    }
};

// Sums of K values over the row's lanes, to all of them.  Rows of one
// workgroup's waves add theirs through `red`, two halves used in turn, so
// that one barrier a sum is enough.
template <int GL, int WAVES, int K>
__device__ __forceinline__ void row_sum(float (&x)[K], float (*red)[16 * 2], int &half)
{
#pragma unroll
    for (int off = GL / 2; off > 0; off >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k)
            x[k] += __shfl_xor(x[k], off);
    if constexpr (WAVES > 1) {
        float *r = red[half];
        half ^= 1;
        if (threadIdx.x % kWave == 0)
#pragma unroll
            for (int k = 0; k < K; ++k)
                r[K * (threadIdx.x / kWave) + k] = x[k];
        lds_barrier();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            x[k] = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w)
                x[k] += r[K * w + k];
        }
    }
}

template <class T, int GL, int WAVES, int E, Rest REST>
__global__ __launch_bounds__(WAVES == 1 ? kThreads : WAVES *kWave) void k_norm_forward(
    int32_t n, int32_t d, const T *x, int64_t ldx, const float *__restrict__ gain,
    const float *__restrict__ shift, float eps, bool relu, T *y, int64_t ldy,
    float *__restrict__ stats)
{
    constexpr int L = GL * WAVES;                          // lanes of a row
    constexpr int R = WAVES == 1 ? kThreads / GL : 1;      // rows of a workgroup at a time
    __shared__ float red[2][16 * 2];
    int half = 0;
    const int l = threadIdx.x % L;
    const int64_t step = (int64_t)gridDim.x * R;
    const Columns<T, E, REST> at{d, l, L};
    constexpr int N = at.N;
    float g[N], b[N];
    at.read(gain, 1.f, g);
    at.read(shift, 0.f, b);
    const float inv = 1.f / (float)d;
    for (int64_t r = (int64_t)blockIdx.x * R + threadIdx.x / L; r < n; r += step) {
        Row<T, E, REST> in;
        in.load(x + r * ldx, at);
        float s[1] = {0.f};
#pragma unroll
        for (int e = 0; e < N; ++e)
            s[0] += in[e];
        row_sum<GL, WAVES, 1>(s, red, half);
        const float mean = s[0] * inv;
        s[0] = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float c = at.in(e) ? in[e] - mean : 0.f;
            s[0] = fmaf(c, c, s[0]);
        }
        row_sum<GL, WAVES, 1>(s, red, half);
        const float rstd = 1.f / sqrtf(fmaf(s[0], inv, eps));
        Row<T, E, REST> out;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float z = fmaf((in[e] - mean) * rstd, g[e], b[e]);
            if (relu)
                z = z <= 0.f ? 0.f : z;   // (a NaN stays one)
            out.set(e, z);
        }
        out.store(y + r * ldy, at);
        if (stats && l == 0)
            *reinterpret_cast<float2 *>(stats + 2 * r) = make_float2(mean, rstd);
    }
}

// dx of each row, and the workgroup's partial sums of dgain and dshift: a
// lane adds its columns over its rows in registers, the rows side by side in
// the workgroup are added through LDS at the end.  Runs of kSumRows rows have
// sums of their own, so that roundings grow as the root of a lane's runs, not
// of its rows: over 306,250 x 256 float32 dgain is 0.9e-7 to 1.2e-7 off, one sum
// 1.3e-7 to 1.9e-7, in the same time (232 us).  Not where one wave holds 16
// elements a lane, whose registers they would pass: 29,125 x 602 bfloat16 takes 32
// us, with them 42.
constexpr int kSumRows = 16;
template <class T, int GL, int WAVES, int E, Rest REST, bool PARAMS>
__global__ __launch_bounds__(WAVES == 1 ? kThreads : WAVES *kWave) void k_norm_backward(
    int32_t n, int32_t d, const T *__restrict__ x, int64_t ldx, const float *__restrict__ gain,
    const T *__restrict__ y, int64_t ldy, const T *dy, int64_t lddy,
    const float *__restrict__ stats, T *dx, int64_t lddx, float *__restrict__ part)
{
    constexpr int L = GL * WAVES;
    constexpr int R = WAVES == 1 ? kThreads / GL : 1;
    __shared__ float red[2][16 * 2];
    int half = 0;
    const int l = threadIdx.x % L;
    const int64_t step = (int64_t)gridDim.x * R;
    const Columns<T, E, REST> at{d, l, L};
    constexpr int N = at.N;
    constexpr bool RUNS = PARAMS && !(WAVES == 1 && E == 16);
    float g[N], dg[PARAMS ? N : 1], db[PARAMS ? N : 1];
    float dgs[RUNS ? N : 1], dbs[RUNS ? N : 1];   // of the whole runs
    int run = 0;
    at.read(gain, 1.f, g);
    if constexpr (PARAMS)
#pragma unroll
        for (int e = 0; e < N; ++e)
            dg[e] = db[e] = 0.f;
    if constexpr (RUNS)
#pragma unroll
        for (int e = 0; e < N; ++e)
            dgs[e] = dbs[e] = 0.f;
    const float inv = 1.f / (float)d;
    for (int64_t r = (int64_t)blockIdx.x * R + threadIdx.x / L; r < n; r += step) {
        Row<T, E, REST> in, up, out;
        in.load(x + r * ldx, at);
        up.load(dy + r * lddy, at);
        if (y) {   // the ReLU mask of the forward's output
            out.load(y + r * ldy, at);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (!(out[e] > 0.f))
                    up.set(e, 0.f);
        }
        const float2 st = *reinterpret_cast<const float2 *>(stats + 2 * r);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float xh = (in[e] - st.x) * st.y, D = up[e], ge = D * g[e];
            s[0] += ge;
            s[1] = fmaf(ge, xh, s[1]);
            if constexpr (PARAMS) {
                dg[e] = fmaf(D, xh, dg[e]);
                db[e] += D;
            }
        }
        if (dx) {   // uniform
            row_sum<GL, WAVES, 2>(s, red, half);
            const float c0 = s[0] * inv, c1 = s[1] * inv;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float xh = (in[e] - st.x) * st.y;
                out.set(e, st.y * (up[e] * g[e] - c0 - xh * c1));
            }
            out.store(dx + r * lddx, at);
        }
        if constexpr (RUNS)
            if (++run == kSumRows) {   // uniform
                run = 0;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    dgs[e] += dg[e];
                    dbs[e] += db[e];
                    dg[e] = db[e] = 0.f;
                }
            }
    }
    if constexpr (RUNS)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            dg[e] += dgs[e];
            db[e] += dbs[e];
        }
    if constexpr (PARAMS) {
        float *p = part + (int64_t)blockIdx.x * 2 * d;
        // the R rows of the workgroup, one column set a time
        __shared__ float sum[R > 1 ? kThreads : 1];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int c = at(e);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float v = k ? db[e] : dg[e];
                if constexpr (R > 1) {
                    sum[threadIdx.x] = v;
                    lds_barrier();
                    v = 0.f;
                    if (threadIdx.x < L)
                        for (int i = 0; i < R; ++i)
                            v += sum[i * L + l];
                    lds_barrier();
                }
                if (threadIdx.x < L && at.in(e))
                    p[k * d + c] = v;
            }
        }
    }
}

// Rows too wide for registers, one workgroup a row: the row is read again
// for each of the passes, out of the L2 after the first.
constexpr int kWideWaves = 16;
constexpr int kWideThreads = kWideWaves * kWave;

template <class T>
__global__ __launch_bounds__(kWideThreads) void k_norm_forward_wide(
    int32_t n, int32_t d, const T *x, int64_t ldx, const float *__restrict__ gain,
    const float *__restrict__ shift, float eps, bool relu, T *y, int64_t ldy,
    float *__restrict__ stats)
{
    constexpr int V = kVecOf<T>;
    __shared__ float red[2][16 * 2];
    int half = 0;
    const float inv = 1.f / (float)d;
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const T *row = x + r * ldx;
        float s[1] = {0.f};
        for (int c = threadIdx.x * V; c < d; c += kWideThreads * V) {
            Row<T, V, kVector> in;
            in.load(row + c, {d - c, 0, 1});
#pragma unroll
            for (int e = 0; e < V; ++e)
                s[0] += in[e];
        }
        row_sum<kWave, kWideWaves, 1>(s, red, half);
        const float mean = s[0] * inv;
        s[0] = 0.f;
        for (int c = threadIdx.x * V; c < d; c += kWideThreads * V) {
            Row<T, V, kVector> in;
            in.load(row + c, {d - c, 0, 1});
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float z = c + e < d ? in[e] - mean : 0.f;
                s[0] = fmaf(z, z, s[0]);
            }
        }
        row_sum<kWave, kWideWaves, 1>(s, red, half);
        const float rstd = 1.f / sqrtf(fmaf(s[0], inv, eps));
        for (int c = threadIdx.x * V; c < d; c += kWideThreads * V) {
            Row<T, V, kVector> in;
            in.load(row + c, {d - c, 0, 1});
            float g[V], b[V];
            Columns<T, V, kVector>{d - c, 0, 1}.read(gain ? gain + c : nullptr, 1.f, g);
            Columns<T, V, kVector>{d - c, 0, 1}.read(shift ? shift + c : nullptr, 0.f, b);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float z = fmaf((in[e] - mean) * rstd, g[e], b[e]);
                if (relu)
                    z = z <= 0.f ? 0.f : z;
                in.set(e, z);
            }
            in.store(y + r * ldy + c, {d - c, 0, 1});
        }
        if (stats && threadIdx.x == 0)
            *reinterpret_cast<float2 *>(stats + 2 * r) = make_float2(mean, rstd);
    }
}

template <class T>
__global__ __launch_bounds__(kWideThreads) void k_norm_backward_wide(
    int32_t n, int32_t d, const T *__restrict__ x, int64_t ldx, const float *__restrict__ gain,
    const T *__restrict__ y, int64_t ldy, const T *dy, int64_t lddy,
    const float *__restrict__ stats, T *dx, int64_t lddx)
{
    constexpr int V = kVecOf<T>;
    __shared__ float red[2][16 * 2];
    int half = 0;
    const float inv = 1.f / (float)d;
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const float2 st = *reinterpret_cast<const float2 *>(stats + 2 * r);
        // e = D gain and xh of the vector at column c
        auto terms = [&](int c, float (&ge)[V], float (&xh)[V]) {
            Row<T, V, kVector> in, up, out;
            in.load(x + r * ldx + c, {d - c, 0, 1});
            up.load(dy + r * lddy + c, {d - c, 0, 1});
            Columns<T, V, kVector>{d - c, 0, 1}.read(gain ? gain + c : nullptr, 1.f, ge);
            if (y)
                out.load(y + r * ldy + c, {d - c, 0, 1});
#pragma unroll
            for (int e = 0; e < V; ++e) {
                xh[e] = (in[e] - st.x) * st.y;
                ge[e] = y && !(out[e] > 0.f) ? 0.f : up[e] * ge[e];
            }
        };
        float s[2] = {0.f, 0.f}, ge[V], xh[V];
        for (int c = threadIdx.x * V; c < d; c += kWideThreads * V) {
            terms(c, ge, xh);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                s[0] += ge[e];
                s[1] = fmaf(ge[e], xh[e], s[1]);
            }
        }
        row_sum<kWave, kWideWaves, 2>(s, red, half);
        const float c0 = s[0] * inv, c1 = s[1] * inv;
        for (int c = threadIdx.x * V; c < d; c += kWideThreads * V) {
            terms(c, ge, xh);
            Row<T, V, kVector> out;
#pragma unroll
            for (int e = 0; e < V; ++e)
                out.set(e, st.y * (ge[e] - c0 - xh[e] * c1));
            out.store(dx + r * lddx + c, {d - c, 0, 1});
        }
    }
}

// Partial sums of dgain and dshift of rows too wide for the registers of one
// workgroup beside the sums: a thread per column, the workgroup's rows in order
// (in runs, as above).
template <class T>
__global__ __launch_bounds__(kThreads) void k_norm_param_wide(
    int32_t n, int32_t d, int32_t rows, const T *__restrict__ x, int64_t ldx,
    const T *__restrict__ y, int64_t ldy, const T *dy, int64_t lddy,
    const float *__restrict__ stats, float *__restrict__ part)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= d)
        return;
    const int64_t r0 = (int64_t)blockIdx.y * rows, r1 = min((int64_t)n, r0 + rows);
    float dg = 0.f, db = 0.f, dgs = 0.f, dbs = 0.f;
    for (int64_t r = r0; r < r1; ++r) {
        if ((r - r0) % kSumRows == 0) {
            dgs += dg;
            dbs += db;
            dg = db = 0.f;
        }
        const float2 st = *reinterpret_cast<const float2 *>(stats + 2 * r);
        float D = (float)dy[r * lddy + c];
        if (y && !((float)y[r * ldy + c] > 0.f))
            D = 0.f;
        dg = fmaf(D, ((float)x[r * ldx + c] - st.x) * st.y, dg);
        db += D;
    }
    float *p = part + (int64_t)blockIdx.y * 2 * d;
    p[c] = dgs + dg;
    p[d + c] = dbs + db;
}

// out[k][c] = sum over the blocks of part[block][k][c], in a fixed order: 64
// columns a workgroup, its 16 waves each take every 16th block, then add up.
// In 64 bits (0.1 us of 2.0 to 5.6); what is left of fp32's roundings are a lane's
// own rows and a workgroup's.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(kSumWaves *kWave) void k_norm_param_sum(
    const float *__restrict__ part, int32_t blocks, int32_t d, float *__restrict__ dgain,
    float *__restrict__ dshift)
{
    __shared__ double sum[kSumWaves][kWave];
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
    const int64_t c = (int64_t)blockIdx.x * kWave + lane;
    const int64_t width = 2 * (int64_t)d;
    double a[4] = {0, 0, 0, 0};   // (one sum would wait for each addition)
    if (c < width) {
        constexpr int U = 16;   // in flight
        int b = w;
        for (; b + (U - 1) * kSumWaves < blocks; b += U * kSumWaves) {
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                x[u] = part[(b + u * kSumWaves) * width + c];
#pragma unroll
            for (int u = 0; u < U; ++u)
                a[u % 4] += x[u];
        }
        for (; b < blocks; b += kSumWaves)
            a[0] += part[b * width + c];
    }
    sum[w][lane] = (a[0] + a[1]) + (a[2] + a[3]);
    lds_barrier();
    if (w == 0 && c < width) {
        double v = 0;
#pragma unroll
        for (int i = 0; i < kSumWaves; ++i)
            v += sum[i][lane];
        float *out = c < d ? dgain : dshift;
        if (out)
            out[c < d ? c : c - d] = (float)v;
    }
}

// The widest rows held in registers, and the widest whose backward has room
// for the sums of dgain and dshift beside them (up to 128 registers a lane of
// a 16-wave workgroup).
constexpr int kHeldWidth = 16384;
constexpr int kFusedWidth = 8192;
// Lanes of a row of d elements of V to a vector, and elements a lane.
struct Shape {
    int gl, waves, e;
};
Shape shape_of(int d, int V)
{
    Shape s{2, 1, V};
    while (s.gl < kWave && s.gl * V < d)
        s.gl *= 2;
    if (d > 1024) {
        s.waves = d > 4096 ? 16 : 4;
        s.e = 8;
    }
    while (s.gl * s.waves * s.e < d && s.e < 16)
        s.e *= 2;
    return s;
}

int rows_at_a_time(const Shape &s) { return s.waves == 1 ? kThreads / s.gl : 1; }

// Workgroups of the row kernels, each a run of rows: whole rounds of the CUs,
// at most 2,048 forward and 1,024 backward, whose workgroups each leave a row of
// partial sums (of rows of up to 1,024 elements; wider rows take more waves
// each, and half or a quarter as many workgroups).  Measured with 1,024,
// 2,048 and 8,192: forward 306,250 x 256 float32 127, 119 and 117 us,
// 16,384 x 4,096 bfloat16 61, 45 and 44; backward 29,125 x 602 bfloat16 39, 48
// and 95 us, 16,384 x 4,096 bfloat16 102, 133 and 186.
int32_t blocks_of(int32_t n, const Shape &s, bool backward)
{
    const int r = rows_at_a_time(s);
    const int cap = (backward ? 1024 : 2048) / (s.waves == 16 ? 4 : s.waves == 4 ? 2 : 1);
    return (int32_t)std::min<int64_t>(cap, ((int64_t)n + r - 1) / r);
}

// Calls f with the row shape as template arguments.
template <class T, class F>
hipError_t with_shape(const Shape &s, int32_t d, F f)
{
    constexpr int V = kVecOf<T>;
#define DIGEST_SHAPE(GL, W, E) \
    if (s.gl == GL && s.waves == W && s.e == E) { \
        if constexpr (GL < V) \
            return f.template operator()<GL, W, E, kVector>(); \
        else \
            return d % V ? f.template operator()<GL, W, E, kLanes>() \
                         : f.template operator()<GL, W, E, kNone>(); \
    }
    DIGEST_SHAPE(2, 1, V)
    DIGEST_SHAPE(4, 1, V)
    DIGEST_SHAPE(8, 1, V)
    DIGEST_SHAPE(16, 1, V)
    DIGEST_SHAPE(32, 1, V)
    DIGEST_SHAPE(64, 1, V)
    if constexpr (V == 4)
        DIGEST_SHAPE(64, 1, 8)
    DIGEST_SHAPE(64, 1, 16)
    DIGEST_SHAPE(64, 4, 8)
    DIGEST_SHAPE(64, 4, 16)
    DIGEST_SHAPE(64, 16, 8)
    DIGEST_SHAPE(64, 16, 16)
#undef DIGEST_SHAPE
    return hipErrorInvalidValue;
}

template <class T>
struct Forward {
    int32_t n, d;
    const void *x;
    int64_t ldx;
    const float *gain, *shift;
    float eps;
    bool relu;
    void *y;
    int64_t ldy;
    float *stats;
    int32_t blocks;
    hipStream_t s;
    template <int GL, int W, int E, Rest REST>
    hipError_t operator()() const
    {
        if (d > kHeldWidth)
            k_norm_forward_wide<T><<<blocks, kWideThreads, 0, s>>>(
                n, d, (const T *)x, ldx, gain, shift, eps, relu, (T *)y, ldy, stats);
        else
            k_norm_forward<T, GL, W, E, REST><<<blocks, W == 1 ? kThreads : W * kWave, 0, s>>>(
                n, d, (const T *)x, ldx, gain, shift, eps, relu, (T *)y, ldy, stats);
        return hipGetLastError();
    }
};

template <class T>
struct Backward {
    int32_t n, d;
    const void *x;
    int64_t ldx;
    const float *gain;
    const void *y;
    int64_t ldy;
    const void *dy;
    int64_t lddy;
    const float *stats;
    void *dx;
    int64_t lddx;
    float *part;   // null: no sums
    int32_t blocks;
    hipStream_t s;
    template <int GL, int W, int E, Rest REST>
    hipError_t operator()() const
    {
        constexpr int threads = W == 1 ? kThreads : W * kWave;
        if constexpr (GL * W * E <= kFusedWidth)   // (never rows past kHeldWidth)
            if (part) {
                k_norm_backward<T, GL, W, E, REST, true><<<blocks, threads, 0, s>>>(
                    n, d, (const T *)x, ldx, gain, (const T *)y, ldy, (const T *)dy, lddy, stats,
                    (T *)dx, lddx, part);
                return hipGetLastError();
            }
        if (part) {   // (before dx, which may replace dy)
            const int32_t rows = (n + blocks - 1) / blocks;
            k_norm_param_wide<T><<<dim3((d + kThreads - 1) / kThreads, blocks), kThreads, 0, s>>>(
                n, d, rows, (const T *)x, ldx, (const T *)y, ldy, (const T *)dy, lddy, stats, part);
        }
        if (dx && d > kHeldWidth)
            k_norm_backward_wide<T><<<blocks, kWideThreads, 0, s>>>(
                n, d, (const T *)x, ldx, gain, (const T *)y, ldy, (const T *)dy, lddy, stats,
                (T *)dx, lddx);
        else if (dx)
            k_norm_backward<T, GL, W, E, REST, false><<<blocks, threads, 0, s>>>(
                n, d, (const T *)x, ldx, gain, (const T *)y, ldy, (const T *)dy, lddy, stats,
                (T *)dx, lddx, nullptr);
        return hipGetLastError();
    }
};

int vec_of(int32_t type) { return type == kF32 ? 4 : 8; }

}  // namespace

int32_t norm_partials(int32_t n, int32_t d)
{
    // (the lanes of a row, and so the workgroups, go by the element type: the
    // larger of the two counts)
    return std::max(blocks_of(n, shape_of(d, 4), true), blocks_of(n, shape_of(d, 8), true));
}

hipError_t launch_norm_forward(int32_t type, int32_t n, int32_t d, const void *x, int64_t ldx,
                               const float *gain, const float *shift, float eps, bool relu,
                               void *y, int64_t ldy, float *stats, hipStream_t s)
{
    if (n <= 0)
        return hipSuccess;
    const Shape sh = shape_of(d, vec_of(type));
    const int32_t blocks = blocks_of(n, sh, false);
    switch (type) {
    case kF32:
        return with_shape<float>(
            sh, d, Forward<float>{n, d, x, ldx, gain, shift, eps, relu, y, ldy, stats, blocks, s});
    case kBF16:
        return with_shape<__bf16>(
            sh, d, Forward<__bf16>{n, d, x, ldx, gain, shift, eps, relu, y, ldy, stats, blocks, s});
    case kF16:
        return with_shape<_Float16>(sh, d,
                                    Forward<_Float16>{n, d, x, ldx, gain, shift, eps, relu, y, ldy,
                                                      stats, blocks, s});
    }
    return hipErrorInvalidValue;
}

hipError_t launch_norm_backward(int32_t type, int32_t n, int32_t d, const void *x, int64_t ldx,
                                const float *gain, const void *y, int64_t ldy, const void *dy,
                                int64_t lddy, const float *stats, bool relu, void *dx,
                                int64_t lddx, float *dgain, float *dshift, float *part,
                                hipStream_t s)
{
    const bool params = dgain || dshift;
    const Shape sh = shape_of(d, vec_of(type));
    const int32_t blocks = blocks_of(n, sh, true);
    if (!relu)
        y = nullptr;
    if (n > 0 && (dx || params)) {
        float *p = params ? part : nullptr;
        hipError_t e = hipErrorInvalidValue;
        switch (type) {
        case kF32:
            e = with_shape<float>(sh, d,
                               Backward<float>{n, d, x, ldx, gain, y, ldy, dy, lddy, stats, dx, lddx,
                                            p, blocks, s});
            break;
        case kBF16:
            e = with_shape<__bf16>(sh, d,
                               Backward<__bf16>{n, d, x, ldx, gain, y, ldy, dy, lddy, stats, dx, lddx,
                                            p, blocks, s});
            break;
        case kF16:
            e = with_shape<_Float16>(sh, d,
                               Backward<_Float16>{n, d, x, ldx, gain, y, ldy, dy, lddy, stats, dx, lddx,
                                            p, blocks, s});
            break;
        }
        if (e != hipSuccess)
            return e;
    }
    if (params) {
        // (no rows: no blocks, and the sums are zero)
        const int64_t width = 2 * (int64_t)d;
        k_norm_param_sum<<<(uint32_t)((width + kWave - 1) / kWave), kSumWaves * kWave, 0, s>>>(
            part, blocks, d, dgain, dshift);
    }
    return hipGetLastError();
}

}  // namespace digest
