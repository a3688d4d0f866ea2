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
// fp32 instructions' peak rate (3 times, by large library products of either).
// The error of five steps against 64 bits is 0.7e-6 to 1.5e-6 of the result
// from 8 x 8 to 2,048 x 2,048 (3.3e-6 at 4,096 x 4,096), that of fp32 products
// 0.5e-6 to 4.2e-6.  A and B are symmetric: only
// the tiles on and above the diagonal are computed, each stored twice.
//
// Large products are bound by the matrix instructions at the clock that the
// card's power allows (4,096 x 4,096: 57% of the cycles at 1.8 GHz; a library
// fp16 product of the same data runs at the same rate), small ones by what a
// dependent launch takes (4 to 5 us of which 1.6 are empty).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "device.h"
#include "train_kernels.h"

namespace digest {
namespace {

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;
constexpr int kBlockK = 32;   // k of one line of LDS

// The wave's number in its workgroup, in a scalar register.
__device__ __forceinline__ int wave_id()
{
    return __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
}

// Where a plane keeps (row, k), k a multiple of 8: the eight values from there
// on lie side by side, 16 bytes of the matrix instruction's operand, in the
// order of its lanes: [row / 32][k / 16][part][k / 8 % 2][row % 32][8].  The
// part (high, low) is kPart further, a block of 32 rows pitch * 64 fp16.
constexpr int kPart = 512;
__device__ __forceinline__ int64_t plane_at(int64_t row, int32_t pitch, int k)
{
    return (row / 32 * pitch + k / 16 * 16) * 64 + (k / 8 % 2) * 256 + row % 32 * 8;
}

// ---------------------------------------------------------------------------
// The update's matrix U and its norm
// ---------------------------------------------------------------------------

// The sum of v over a workgroup of THREADS, to all its threads, in a fixed order.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double sum[THREADS / kWave];
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1)
        v += __shfl_xor(v, off);
    if (threadIdx.x % kWave == 0)
        sum[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w)
        v += sum[w];
    return v;
}

// Runs of kOrthSumRun elements of a matrix, one vector of four a thread:
// f(element index, count) for each thread's vectors; the matrix's rows one
// after another where they are contiguous, else each row's runs.  (With
// four a thread they came one after another: the momenta of a 100-256-256-47
// network from eight gradients 8.4 us, now 4.8; of six matrices of 1,024 x
// 1,024 to 4,096 34 to 35 either way.)
constexpr int kRunVec = 4;
static_assert(kOrthSumRun == kThreads * kRunVec, "a run is one vector a thread");
template <class F>
__device__ __forceinline__ void for_vectors(const OrthItem &it, int64_t ld, F f)
{
    constexpr int V = kRunVec;
    const bool flat = ld == it.cols;
    const int64_t len = flat ? (int64_t)it.rows * it.cols : it.cols;
    const int64_t runs = (len + kOrthSumRun - 1) / kOrthSumRun;
    for (int64_t q = blockIdx.x; q < runs * (flat ? 1 : it.rows); q += it.sums) {
        const int64_t row = flat ? 0 : q / runs, from = (q - row * runs) * kOrthSumRun;
        const int64_t at = from + (int)threadIdx.x * V;
        if (at < len)
            f(row * ld + at, (int)min((int64_t)V, len - at));
    }
}

template <class T, int V>
struct Vec {
    typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
// n <= V elements at p, zeros behind them.
template <class T, int V>
__device__ __forceinline__ typename Vec<T, V>::type load_some(const T *p, int n)
{
    typedef typename Vec<T, V>::type vec;
    if (n == V)
        return *reinterpret_cast<const vec *>(p);
    vec v;
#pragma unroll
    for (int j = 0; j < V; ++j)
        v[j] = j < n ? p[j] : (T)0.f;
    return v;
}
template <class T, int V>
__device__ __forceinline__ void store_some(T *p, int n, typename Vec<T, V>::type v)
{
    if (n == V) {
        *reinterpret_cast<typename Vec<T, V>::type *>(p) = v;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < n)
                p[j] = v[j];
    }
}

// Partial sums of the squares of U, 64 bits: their range holds the squares of
// every fp32 number.
template <class T>
__global__ __launch_bounds__(kThreads) void k_orth_sum(OrthBatch b)
{
    constexpr int V = kRunVec;
    const OrthItem &it = b.item[blockIdx.y];
    if ((int)blockIdx.x >= it.sums)
        return;
    double v = 0;
    for_vectors(it, it.ldu, [&](int64_t at, int n) {
        const auto x = load_some<T, V>((const T *)it.u + at, n);
#pragma unroll
        for (int j = 0; j < V; ++j)
            v += (double)(float)x[j] * (double)(float)x[j];
    });
    v = block_sum<kThreads>(v);
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
    const float inv = 1.f / (float)per_item;
    double v = 0;
    for_vectors(it, it.cols, [&](int64_t at, int n) {
        auto mo = load_some<float, 4>(it.mom + at, n);
        auto s = load_some<float, 4>(g[0] + at, n);
        int m = 1;
        for (; m + 4 <= per_item; m += 4) {   // four in flight, added in order
            Vec<float, 4>::type x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[j] = load_some<float, 4>(g[m + j] + at, n);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                s += x[j];
        }
        for (; m < per_item; ++m)
            s += load_some<float, 4>(g[m] + at, n);
        auto x = s;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float mean = s[j] * inv;
            mo[j] = fmaf(beta, mo[j], mean);
            x[j] = nesterov ? fmaf(beta, mo[j], mean) : mo[j];
            if (j < n)
                v += (double)x[j] * (double)x[j];
        }
        store_some<float, 4>(it.mom + at, n, mo);
        store_some<float, 4>(u + at, n, x);
    });
    v = block_sum<kThreads>(v);
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
    *reinterpret_cast<half8 *>(dst + kPart) = l;
}

template <class T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_orth_split(OrthBatch b, double scale)
{
    __shared__ float tile[kSplitTile][kSplitTile + 1];
    const OrthItem &it = b.item[blockIdx.z];
    const bool tall = it.rows > it.cols;
    const int i0 = blockIdx.y * kSplitTile, j0 = blockIdx.x * kSplitTile;
    // padded extents of U's rows and columns
    if (i0 >= (tall ? it.cp : it.rp) || j0 >= (tall ? it.rp : it.cp))
        return;
    const T *u = (const T *)it.u;
    constexpr int N = kSplitTile * kSplitTile / THREADS;
    const int tj = threadIdx.x % kSplitTile, t0 = threadIdx.x / kSplitTile;
    float x[N];   // (on their way while the norm is formed)
#pragma unroll
    for (int q = 0; q < N; ++q) {
        const int i = i0 + t0 + q * (THREADS / kSplitTile), j = j0 + tj;
        x[q] = i < it.rows && j < it.cols ? (float)u[(int64_t)i * it.ldu + j] : 0.f;
    }
    double sum = 0;
    if (it.sums <= kWave) {   // (uniform; every wave adds them itself)
        if ((int)threadIdx.x % kWave < it.sums)
            sum = it.part[threadIdx.x % kWave];
#pragma unroll
        for (int off = kWave / 2; off > 0; off >>= 1)
            sum += __shfl_xor(sum, off);
    } else {
        for (int i = threadIdx.x; i < it.sums; i += THREADS)
            sum += it.part[i];
        sum = block_sum<THREADS>(sum);
    }
    const double norm = sqrt(sum);
    const double f = norm == 0 ? 0.0 : scale / norm;
#pragma unroll
    for (int q = 0; q < N; ++q)
        tile[t0 + q * (THREADS / kSplitTile)][tj] = (float)((double)x[q] * f);
    __syncthreads();
    _Float16 *p = (_Float16 *)(tall ? it.Xt[0] : it.X);
    _Float16 *pt = (_Float16 *)(tall ? it.X : it.Xt[0]);
    const int kp = tall ? it.rk : it.ck, kt = tall ? it.ck : it.rk;
    for (int q = threadIdx.x; q < kSplitTile * kSplitTile / 8; q += THREADS) {
        const int row = q % kSplitTile, k = q / kSplitTile * 8;   // (rows side by side)
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
constexpr bool symmetric(int mode) { return mode == kGram || mode == kPoly; }

constexpr int kLineBytes = 4096;   // 32 rows, 32 k, both parts

struct OrthParams {
    float alpha;         // plane products to the stored value's scale
    float diag, lin;     // kPoly: a 2^eb, b 2^(eb - ea)
    float keep;
    int32_t from;
    // Workgroups: the whole tiles [0, whole), then the parts of the others
    // (chunk lines of k each, item i's parts from work0[i] on).
    int32_t whole, chunk;
    int32_t tile0[kOrthItems + 1], work0[kOrthItems], parts[kOrthItems];
    float *partials;
};

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

// The item whose range of `first` (ascending; entries past the last item are
// beyond every v) holds v: all of it read at once, no search.
__device__ __forceinline__ int item_of(const int32_t *first, int v)
{
    int i = 0;
#pragma unroll
    for (int j = 1; j < kOrthItems; ++j)
        i += v >= first[j];
    return i;
}

template <int MODE>
__device__ __forceinline__ void operands(const OrthItem &it, const OrthParams &pr, int &K,
                                         const char *&P, const char *&Q)
{
    K = MODE == kGram ? it.ck : it.rk;
    P = (const char *)(MODE == kGram ? it.X : MODE == kPoly ? it.A : it.B);
    Q = (const char *)(MODE == kGram ? it.X : MODE == kPoly ? it.A : it.Xt[pr.from]);
}

// Tile t of an item, TILE x TILE.  Symmetric products: the tiles on and above
// the diagonal, by column.
template <bool SYM, int TILE>
__device__ __forceinline__ void tile_of(int rp, int t, int &tm, int &tn)
{
    if constexpr (SYM) {
        tn = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
        while (tn * (tn + 1) / 2 > t)
            --tn;
        while ((tn + 1) * (tn + 2) / 2 <= t)
            ++tn;
        tm = t - tn * (tn + 1) / 2;
    } else {
        const int gm = (rp + TILE - 1) / TILE;
        tm = t % gm;
        tn = t / gm;
    }
}
int32_t tiles_of(const OrthItem &it, bool sym, int tile)
{
    const int32_t gm = (it.rp + tile - 1) / tile;
    return sym ? gm * (gm + 1) / 2 : gm * ((it.cp + tile - 1) / tile);
}

// Rows m .. m + N - 1 of column n of the result, into the caller's matrix or
// (UPDATE) into the weights: out <- keep out - scale v, all of them read
// before the first is written.
template <bool UPDATE, int N, class T>
__device__ __forceinline__ void put_result(const OrthItem &it, float keep, int m, int n,
                                           const float (&v)[N], T *out)
{
    const int count = n < it.c ? max(0, min(N, it.r - m)) : 0;
    if (it.rows > it.cols) {   // (tall: side by side)
        T *o = out + (int64_t)n * it.ldo + m;
        typename Vec<T, N>::type x;
        if constexpr (UPDATE)
            x = load_some<T, N>(o, count);
#pragma unroll
        for (int e = 0; e < N; ++e)
            x[e] = (T)(UPDATE ? keep * (float)x[e] - it.scale * v[e] : v[e]);
        store_some<T, N>(o, count, x);
    } else {
        T *o = out + (int64_t)m * it.ldo + n, x[N];
        if constexpr (UPDATE)
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (e < count)
                    x[e] = o[e * it.ldo];
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < count)
                o[e * it.ldo] = (T)(UPDATE ? keep * (float)x[e] - it.scale * v[e] : v[e]);
    }
}

// Stores 32 columns n from nb on and 16 rows m from mb on of the product,
// given by rows: lane (n = lane % 32, lane / 32) holds m = 8 (lane / 32) ..
// + 7.  `mirror`: the transposed is nobody else's to store.  `turn` is the
// wave's own LDS.
constexpr int kTurn = 32 * 20;
// kPoly's elements of A there: A is symmetric, row n holds the eight side by side.
struct Eights {
    half8 h, l;
    __device__ __forceinline__ void load(const OrthItem &it, int mb, int nb)
    {
        const int lane = threadIdx.x % kWave;
        const _Float16 *a = (const _Float16 *)it.A +
                            plane_at(nb + lane % 32, it.rk, mb + lane / 32 * 8);
        h = *reinterpret_cast<const half8 *>(a);
        l = *reinterpret_cast<const half8 *>(a + kPart);
    }
};
template <int MODE, class T>
__device__ __forceinline__ void put(const OrthItem &it, const OrthParams &pr, int mb, int nb,
                                    float (&v)[8], const Eights &a, bool mirror, uint32_t *turn)
{
    const int lane = threadIdx.x % kWave;
    const int m = mb + lane / 32 * 8, n = nb + lane % 32;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] *= pr.alpha;
    if constexpr (MODE == kPoly) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = fmaf((float)a.h[e] + (float)a.l[e], pr.lin, v[e]) +
                   (m + e == n ? pr.diag : 0.f);
    }
    if constexpr (MODE == kGram || MODE == kPoly || MODE == kApply) {
        union {
            half8 v;
            uint16_t u[8];
        } h, l;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h.v[e] = (_Float16)v[e];
            l.v[e] = (_Float16)(v[e] - (float)h.v[e]);
        }
        _Float16 *d = (_Float16 *)(MODE == kGram ? it.A : MODE == kPoly ? it.B : it.X);
        if (mirror) {
            _Float16 *dt = (symmetric(MODE) ? d : (_Float16 *)it.Xt[pr.from ^ 1]) +
                           plane_at(n, it.rk, m);
            *reinterpret_cast<half8 *>(dt) = h.v;
            *reinterpret_cast<half8 *>(dt + kPart) = l.v;
        }
        // turned over in LDS: lane (m = lane % 16, lane / 16) takes n = 8 (lane / 16) .. + 7
        // (rows 20 words apart)
        uint4 *w = reinterpret_cast<uint4 *>(turn + lane % 32 * 20 + lane / 32 * 8);
#pragma unroll
        for (int e = 0; e < 2; ++e)
            w[e] = make_uint4(h.u[4 * e] | l.u[4 * e] << 16, h.u[4 * e + 1] | l.u[4 * e + 1] << 16,
                              h.u[4 * e + 2] | l.u[4 * e + 2] << 16,
                              h.u[4 * e + 3] | l.u[4 * e + 3] << 16);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        const uint32_t *r = turn + lane / 16 * 160 + lane % 16;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h.u[e] = (uint16_t)r[20 * e];
            l.u[e] = (uint16_t)(r[20 * e] >> 16);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        d += plane_at(mb + lane % 16, symmetric(MODE) ? it.rk : it.ck, nb + lane / 16 * 8);
        *reinterpret_cast<half8 *>(d) = h.v;
        *reinterpret_cast<half8 *>(d + kPart) = l.v;
    } else {
        put_result<MODE == kUpdate, 8>(it, pr.keep, m, n, v, (T *)it.out);
    }
}

// The matrix instruction's 32 x 32 result, lane (n, lane / 32) with rows
// 8 g + 4 (lane / 32) + e in element 4 g + e, to rows as put takes them: 16
// rows of half s.
__device__ __forceinline__ void rows_of(const floatx16 &x, int s, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        // the upper lanes' x[8 s + e] against the lower lanes' x[8 s + 4 + e]
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[8 * s + e]),
                                                        __float_as_uint(x[8 * s + 4 + e]), false,
                                                        false);
        v[e] = __uint_as_float(r[0]);
        v[4 + e] = __uint_as_float(r[1]);
    }
}

// A symmetric product's 32 x 32 block at (mb, nb): blocks below the diagonal
// are the mirror of those above.
template <int MODE>
__device__ __forceinline__ bool stored(int rp, int cp, int mb, int nb)
{
    if (symmetric(MODE))
        return mb <= nb && nb < rp;
    return mb < rp && nb < cp;
}

__device__ __forceinline__ floatx16 zero16()
{
    floatx16 z;
#pragma unroll
    for (int e = 0; e < 16; ++e)
        z[e] = 0.f;
    return z;
}

// The large products: a TILE x TILE tile of D per workgroup and CU, 128 (4
// waves of 64 x 64) or 256 (8 waves of 128 x 64, which read each line of LDS
// and of memory fewer times).  Lines (32 k) of both operands' rows come into a
// ring of BUFS places in LDS.
template <int TILE>
struct Waves {
    static constexpr int WM = 2, WN = TILE / 64, TM = TILE / 64, TN = 2, W = WM * WN;
    static_assert(WN * TN * 32 == TILE && WM * TM * 32 == TILE, "the waves cover the tile");
};
template <int MODE, class T, int TILE>
__global__ __launch_bounds__(Waves<TILE>::W *kWave) void k_orth_gemm(OrthBatch b, OrthParams pr)
{
    constexpr int BUFS = TILE == 128 ? 4 : 2;   // 128 KB either way
    constexpr int WN = Waves<TILE>::WN, TM = Waves<TILE>::TM, TN = Waves<TILE>::TN;
    constexpr int W = Waves<TILE>::W, BM = TILE, BN = TILE, ROWS = (BM + BN) / 32;
    // [32 rows][16 k][part][lane]: what a matrix instruction takes is 1 KB.  A
    // ring of BUFS lines (arrays of their own: the compiler then knows which
    // one a load fills).
    __shared__ half8 lds0[ROWS * kLineBytes / 16], lds1[ROWS * kLineBytes / 16];
    static_assert(BUFS == 2 || BUFS == 4, "places for lines");
    __shared__ half8 lds2[BUFS > 2 ? ROWS * kLineBytes / 16 : 1];
    __shared__ half8 lds3[BUFS > 2 ? ROWS * kLineBytes / 16 : 1];

    int w = blockIdx.x, i, t, part = -1;
    if (w < pr.whole) {
        w = (int)xcd_contiguous(w, pr.whole);
        i = item_of(pr.tile0, w);
        t = w - pr.tile0[i];
    } else {
        i = item_of(pr.work0, w);
        part = (w - pr.work0[i]) % pr.parts[i];
        t = max(pr.whole - pr.tile0[i], 0) + (w - pr.work0[i]) / pr.parts[i];
    }
    const OrthItem &it = b.item[i];
    int tm, tn, K;
    tile_of<symmetric(MODE), TILE>(it.rp, t, tm, tn);
    const char *P, *Q;
    operands<MODE>(it, pr, K, P, Q);
    const int lane = threadIdx.x % kWave, wave = wave_id();
    const int wm = wave / WN * TM, wn = wave % WN * TN;   // in blocks of 32

    // the small products have sums of their own where registers allow, added at
    // the end: the large ones are then rounded a third as often
    constexpr bool TWO = TILE == 128;
    floatx16 acc[TM][TN], low[TWO ? TM : 1][TWO ? TN : 1];
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y) {
            acc[x][y] = zero16();
            if constexpr (TWO)
                low[x][y] = zero16();
        }

    // A wave's instruction takes 1 KB of a line's 4 KB for 32 rows; rows past
    // the operand repeat its last 32 (their products are not stored).
    const int64_t pitch = (int64_t)K * 128;   // bytes of 32 rows
    const int prow = it.rp / 32, qrow = (symmetric(MODE) ? it.rp : it.cp) / 32;
    const uint32_t loff = lane * 16;
    constexpr int L = 4 * ROWS / W;   // its loads of a line
    auto load_one = [&](int kb, half8 *dst, int q) {
        const int at = q * W + wave, row = at / 4;
        const char *src = row < BM / 32
                              ? P + min(tm * (BM / 32) + row, prow - 1) * pitch
                              : Q + min(tn * (BN / 32) + row - BM / 32, qrow - 1) * pitch;
        src += (int64_t)kb * kLineBytes + at % 4 * 1024;
        __builtin_amdgcn_global_load_lds((global_void *)(src + loff),
                                         (lds_void *)(&dst[at * kWave]), 16, 0, 0);
    };
    auto load = [&](int kb, half8 *dst) {
#pragma unroll
        for (int q = 0; q < L; ++q)
            load_one(kb, dst, q);
    };
    struct Frags {   // the operands of 16 k
        half8 p[2][TM], q[2][TN];
    };
    constexpr int F = 2 * (TM + TN);   // reads of a Frags
    auto fetch_one = [&](const half8 *src, int s, Frags &f, int i) {
        const int h = i % 2, x = i / 2;
        if (x < TM)
            f.p[h][x] = src[((wm + x) * 4 + 2 * s + h) * kWave + lane];
        else
            f.q[h][x - TM] = src[((BM / 32 + wn + x - TM) * 4 + 2 * s + h) * kWave + lane];
    };
    // f's products, `beside(i)` issued behind the i-th: reads and loads take
    // their turn while the matrix instructions run
    auto multiply = [&](const Frags &f, auto beside) {
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int x = 0; x < TM; ++x)
#pragma unroll
                for (int y = 0; y < TN; ++y) {
                    floatx16 &d = TWO && k > 0 ? low[TWO ? x : 0][TWO ? y : 0] : acc[x][y];
                    d = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.p[k == 2][x], f.q[k == 1][y], d, 0,
                                                               0, 0);
                    beside((k * TM + x) * TN + y);
                    __builtin_amdgcn_sched_barrier(0);
                }
    };
    static_assert(F <= 3 * TM * TN && L <= 3 * TM * TN, "a place behind a product for each");
    // Waits until all but the wave's newest `lines` lines are in LDS and its
    // reads are done, then for the other waves.  (A barrier of the compiler's
    // would wait for every load.)
    static_assert((BUFS - 1) * L < 64, "vmcnt holds six bits");
    auto sync = [&](auto lines) {
        constexpr int n = decltype(lines)::value * L;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((n & 15) | 7 << 4 | (n >> 4) << 14);
        asm volatile("s_barrier" ::: "memory");
    };
    const int k0 = part < 0 ? 0 : part * pr.chunk;
    const int k1 = part < 0 ? K / kBlockK : min(K / kBlockK, k0 + pr.chunk);
    // One line: its first half is in f0 already.  The second half is read while
    // the first is multiplied, the next line's first half while the second is;
    // between them the line's place in LDS is free for the line BUFS further.
    // (Past the last line it is loaded again, so that the waits count alike.)
    Frags f0, f1;
    auto step = [&](int kb, half8 *now, const half8 *next) {
        __builtin_amdgcn_s_waitcnt(15 | 7 << 4 | 3 << 14);   // f0, before f1 is asked for
        multiply(f0, [&](int i) {
            if (i < F)
                fetch_one(now, 1, f1, i);
        });
        sync(std::integral_constant<int, BUFS - 2>());
        const int further = min(kb + BUFS, k1 - 1);
        multiply(f1, [&](int i) {
            if (i < F)
                fetch_one(next, 0, f0, i);
            if (i < L)
                load_one(further, now, i);
        });
    };
    load(k0, lds0);
    load(min(k0 + 1, k1 - 1), lds1);
    if constexpr (BUFS == 4) {
        load(min(k0 + 2, k1 - 1), lds2);
        load(min(k0 + 3, k1 - 1), lds3);
    }
    sync(std::integral_constant<int, BUFS - 1>());
#pragma unroll
    for (int i = 0; i < F; ++i)
        fetch_one(lds0, 0, f0, i);
    int kb = k0;
    if constexpr (BUFS == 4)
        for (; kb + 4 <= k1; kb += 4) {
            step(kb, lds0, lds1);
            step(kb + 1, lds1, lds2);
            step(kb + 2, lds2, lds3);
            step(kb + 3, lds3, lds0);
        }
    for (; kb < k1; kb += 2) {   // (an even number of lines)
        step(kb, lds0, lds1);
        step(kb + 1, lds1, BUFS == 4 ? lds2 : lds0);
    }
    __syncthreads();

    // (what the stores need is formed here, not kept through the loop)
    int lane_out = lane;
    asm volatile("" : "+v"(lane_out));
    static_assert(sizeof(lds0) >= W * kTurn * 4, "room to turn blocks");
    uint32_t *turn = reinterpret_cast<uint32_t *>(lds0) + wave * kTurn;
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y) {
            const int mb = tm * BM + (wm + x) * 32, nb = tn * BN + (wn + y) * 32;
            if (!stored<MODE>(it.rp, it.cp, mb, nb))
                continue;
            if constexpr (TWO)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    acc[x][y][e] += low[x][y][e];
            if (part < 0) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    float v[8];
                    Eights a;
                    if constexpr (MODE == kPoly)
                        a.load(it, mb + 16 * s, nb);
                    rows_of(acc[x][y], s, v);
                    put<MODE, T>(it, pr, mb + 16 * s, nb, v, a, !symmetric(MODE) || mb != nb, turn);
                }
            } else {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float *d = pr.partials + (int64_t)(w - pr.whole) * (BM * BN) +
                               ((((wave * TM + x) * TN + y) * 4 + g) * kWave + lane_out) * 4;
                    *reinterpret_cast<float4 *>(d) =
                        make_float4(acc[x][y][4 * g], acc[x][y][4 * g + 1], acc[x][y][4 * g + 2],
                                    acc[x][y][4 * g + 3]);
                }
            }
        }
}

// Sums the parts of the tiles that were split, one wave 16 rows of a block.
template <int MODE, class T, int TILE>
__global__ __launch_bounds__(kThreads) void k_orth_join(OrthBatch b, OrthParams pr)
{
    constexpr int WN = Waves<TILE>::WN, TM = Waves<TILE>::TM, TN = Waves<TILE>::TN;
    constexpr int BM = TILE, BN = TILE, UNITS = Waves<TILE>::W * TM * TN * 2;
    __shared__ uint32_t turn[kThreads / kWave][kTurn];
    const int lane = threadIdx.x % kWave;
    const int at = blockIdx.x * (kThreads / kWave) + wave_id();
    const int tile = pr.whole + at / UNITS;
    const int i = item_of(pr.tile0, tile);
    const OrthItem &it = b.item[i];
    const int first = max(pr.whole, pr.tile0[i]);   // the item's first split tile
    int tm, tn;
    tile_of<symmetric(MODE), TILE>(it.rp, tile - pr.tile0[i], tm, tn);
    const int blk = at % UNITS / 2, s = at % 2;
    const int wave = blk / (TM * TN), x = blk / TN % TM, y = blk % TN;
    const int mb = tm * BM + (wave / WN * TM + x) * 32, nb = tn * BN + (wave % WN * TN + y) * 32;
    if (!stored<MODE>(it.rp, it.cp, mb, nb))
        return;
    // rows 8 (lane / 32) .. + 7 of half s: element group 2 s + lane / 32 of both lane halves
    const int part0 = pr.work0[i] - pr.whole + (tile - first) * pr.parts[i];
    const float *src = pr.partials + (int64_t)part0 * (BM * BN) +
                       ((blk * 4 + 2 * s + lane / 32) * kWave + lane % 32) * 4;
    Eights a;
    if constexpr (MODE == kPoly)
        a.load(it, mb + 16 * s, nb);
    float v[8] = {};
    constexpr int U = 8;   // parts in flight
    for (int p0 = 0; p0 < pr.parts[i]; p0 += U) {
        float4 f[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float *q = src + (int64_t)min(p0 + u, pr.parts[i] - 1) * (BM * BN);
            f[u][0] = *reinterpret_cast<const float4 *>(q);
            f[u][1] = *reinterpret_cast<const float4 *>(q + 128);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p0 + u < pr.parts[i]) {
                v[0] += f[u][0].x, v[1] += f[u][0].y, v[2] += f[u][0].z, v[3] += f[u][0].w;
                v[4] += f[u][1].x, v[5] += f[u][1].y, v[6] += f[u][1].z, v[7] += f[u][1].w;
            }
    }
    put<MODE, T>(it, pr, mb + 16 * s, nb, v, a, !symmetric(MODE) || mb != nb, turn[wave_id()]);
}

// The small products, bound by latency: TS x TS blocks of 32 x 32 of D per
// workgroup, whose waves split k among themselves (a line in turn, straight
// from memory into the registers that multiply, DEPTH lines in flight) and
// add their sums through LDS in wave order.
constexpr int kSmallWaves = 8;

template <int MODE, class T, int TS, int DEPTH>
__global__ __launch_bounds__(kSmallWaves *kWave) void k_orth_small(OrthBatch b, OrthParams pr)
{
    constexpr int TILE = 32 * TS, GROUPS = TS * TS * 4, UNITS = TS * TS * 2;
    __shared__ float4 sum[kSmallWaves][GROUPS][kWave];
    __shared__ uint32_t turn[UNITS][kTurn];
    const int w = blockIdx.x, i = item_of(pr.tile0, w);
    const OrthItem &it = b.item[i];
    int tm, tn, K;
    const char *P, *Q;
    operands<MODE>(it, pr, K, P, Q);
    int t = w - pr.tile0[i], rp = it.rp, cp = it.cp;
    // (everything that the loads need is fetched here, at once)
    asm volatile("" : "+s"(K), "+s"(P), "+s"(Q), "+s"(t), "+s"(rp), "+s"(cp));
    tile_of<symmetric(MODE), TILE>(rp, t, tm, tn);
    const int lane = threadIdx.x % kWave, wave = wave_id();
    const int64_t pitch = (int64_t)K * 128;
    const uint32_t loff = lane * 16;
    P += tm * TS * pitch;
    Q += tn * TS * pitch;

    // at the end a wave stores 16 rows of a block
    static_assert(UNITS <= kSmallWaves, "a wave for each half of a block");
    const int blk = wave / 2, s = wave % 2;
    const int mb = tm * TILE + blk / TS * 32, nb = tn * TILE + blk % TS * 32;
    const bool stores = wave < UNITS && stored<MODE>(rp, cp, mb, nb);
    Eights a;
    if constexpr (MODE == kPoly)
        if (stores)
            a.load(it, mb + 16 * s, nb);

    constexpr bool TWO = TS == 1;   // (sums of their own for the small products, as above)
    floatx16 acc[TS][TS], low[TWO ? TS : 1][TWO ? TS : 1];
#pragma unroll
    for (int x = 0; x < TS; ++x)
#pragma unroll
        for (int y = 0; y < TS; ++y) {
            acc[x][y] = zero16();
            if constexpr (TWO)
                low[x][y] = zero16();
        }
    struct Line {
        half8 p[2][2][TS], q[2][2][TS];   // [16 k][part][block]
    };
    const int nk = K / kBlockK;
    auto load = [&](int kb, Line &l) {
        if (kb >= nk)   // uniform
            return;
        const int64_t at = (int64_t)kb * kLineBytes;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int x = 0; x < TS; ++x) {
                    const int64_t o = x * pitch + at + (2 * s + h) * 1024;
                    l.p[s][h][x] = *reinterpret_cast<const half8 *>(P + o + loff);
                    l.q[s][h][x] = *reinterpret_cast<const half8 *>(Q + o + loff);
                }
    };
    auto multiply = [&](const Line &l) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll
                for (int x = 0; x < TS; ++x)
#pragma unroll
                    for (int y = 0; y < TS; ++y) {
                        floatx16 &d = TWO && k > 0 ? low[TWO ? x : 0][TWO ? y : 0] : acc[x][y];
                        d = __builtin_amdgcn_mfma_f32_32x32x16_f16(l.p[s][k == 2][x],
                                                                   l.q[s][k == 1][y], d, 0, 0, 0);
                    }
    };
    if (wave < nk) {
        Line l[DEPTH];
#pragma unroll
        for (int u = 0; u < DEPTH; ++u)
            load(wave + u * kSmallWaves, l[u]);
        for (int kb = wave; kb < nk; kb += DEPTH * kSmallWaves) {
#pragma unroll
            for (int u = 0; u < DEPTH; ++u) {
                if (kb + u * kSmallWaves < nk)   // uniform
                    multiply(l[u]);
                load(kb + (u + DEPTH) * kSmallWaves, l[u]);
            }
        }
    }
    const int waves = min(kSmallWaves, nk);   // the others' sums are zero
    if (wave < waves)
#pragma unroll
        for (int x = 0; x < TS; ++x)
#pragma unroll
            for (int y = 0; y < TS; ++y) {
                if constexpr (TWO)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        acc[x][y][e] += low[x][y][e];
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    sum[wave][(TS * x + y) * 4 + g][lane] =
                        make_float4(acc[x][y][4 * g], acc[x][y][4 * g + 1], acc[x][y][4 * g + 2],
                                    acc[x][y][4 * g + 3]);
            }
    __syncthreads();
    if (!stores)
        return;
    float v[8] = {};
    for (int p = 0; p < waves; ++p) {
        const float4 *f = &sum[p][blk * 4 + 2 * s + lane / 32][lane % 32];
        v[0] += f[0].x, v[1] += f[0].y, v[2] += f[0].z, v[3] += f[0].w;
        v[4] += f[32].x, v[5] += f[32].y, v[6] += f[32].z, v[7] += f[32].w;
    }
    put<MODE, T>(it, pr, mb + 16 * s, nb, v, a, !symmetric(MODE) || mb != nb, turn[wave]);
}

// X' = (a I + b A + c A A) X for up to 128 rows, 32 x 32 of X' per workgroup,
// in one launch instead of two: wave j forms B's 32 x 32 block of the tile's
// rows and k in [32 j, 32 j + 32) itself, whose layout as a result is the
// matrix instruction's layout as an operand, and multiplies it by its 32 k of
// X.  The waves' sums meet in LDS.  B is formed again for every 32 columns of
// X: 100 x 256 in five steps takes 52 us for 61 (5.8 us a step here), but
// 256 x 256 (eight waves) 9.5 us a step where B and B X take 4.6 each, so it
// stops at 128.
constexpr int kFuseWaves = 4;
constexpr int kFuseRows = 32 * kFuseWaves;

template <int MODE, class T>
__global__ __launch_bounds__(kFuseWaves *kWave) void k_orth_poly_apply(OrthBatch b, OrthParams poly,
                                                                        OrthParams pr)
{
    __shared__ float4 sum[kFuseWaves][4][kWave];
    __shared__ uint32_t turn[2][kTurn];
    const int w = blockIdx.x, i = item_of(pr.tile0, w);
    const OrthItem &it = b.item[i];
    int K = it.rk, t = w - pr.tile0[i], rp = it.rp;
    const char *A = (const char *)it.A, *Q = (const char *)it.Xt[pr.from];
    // (everything that the loads need is fetched here, at once)
    asm volatile("" : "+s"(K), "+s"(A), "+s"(Q), "+s"(t), "+s"(rp));
    int tm, tn;
    tile_of<false, 32>(rp, t, tm, tn);
    const int lane = threadIdx.x % kWave, wave = wave_id(), nk = K / kBlockK;
    const int64_t pitch = (int64_t)K * 128;
    const uint32_t loff = lane * 16;
    if (wave < nk) {
        half8 x[2][2];   // X's line of the wave's k: [16 k][part]
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                x[s][h] = *reinterpret_cast<const half8 *>(Q + tn * pitch + wave * kLineBytes +
                                                           (2 * s + h) * 1024 + loff);
        Eights a[2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
            a[s].load(it, 32 * wave + 16 * s, 32 * tm);
        const char *p = A + wave * pitch + loff, *q = A + tm * pitch + loff;
        floatx16 acc, low;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            acc[e] = low[e] = 0.f;
        half8 f[kFuseWaves][2][2], g[kFuseWaves][2][2];
#pragma unroll
        for (int k = 0; k < kFuseWaves; ++k)
            if (k < nk)   // uniform
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int64_t o = (int64_t)k * kLineBytes + (2 * s + h) * 1024;
                        f[k][s][h] = *reinterpret_cast<const half8 *>(p + o);
                        g[k][s][h] = *reinterpret_cast<const half8 *>(q + o);
                    }
#pragma unroll
        for (int k = 0; k < kFuseWaves; ++k)
            if (k < nk)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[k][s][0], g[k][s][0], acc, 0, 0,
                                                                 0);
                    low = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[k][s][0], g[k][s][1], low, 0, 0,
                                                                 0);
                    low = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[k][s][1], g[k][s][0], low, 0, 0,
                                                                 0);
                }
#pragma unroll
        for (int e = 0; e < 16; ++e)
            acc[e] += low[e];
        floatx16 out;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            out[e] = 0.f;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            // row n = lane % 32 of the tile, k = m .. m + 7
            float v[8];
            rows_of(acc, s, v);
            const int m = 32 * wave + 16 * s + lane / 32 * 8, n = 32 * tm + lane % 32;
            half8 h, l;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = fmaf((float)a[s].h[e] + (float)a[s].l[e], poly.lin, v[e] * poly.alpha) +
                       (m + e == n ? poly.diag : 0.f);
                h[e] = (_Float16)v[e];
                l[e] = (_Float16)(v[e] - (float)h[e]);
            }
            out = __builtin_amdgcn_mfma_f32_32x32x16_f16(h, x[s][0], out, 0, 0, 0);
            out = __builtin_amdgcn_mfma_f32_32x32x16_f16(h, x[s][1], out, 0, 0, 0);
            out = __builtin_amdgcn_mfma_f32_32x32x16_f16(l, x[s][0], out, 0, 0, 0);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g)
            sum[wave][g][lane] = make_float4(out[4 * g], out[4 * g + 1], out[4 * g + 2],
                                             out[4 * g + 3]);
    }
    __syncthreads();
    if (wave >= 2)
        return;
    // a wave stores 16 rows
    float v[8] = {};
    for (int p = 0; p < nk; ++p) {
        const float4 *f = &sum[p][2 * wave + lane / 32][lane % 32];
        v[0] += f[0].x, v[1] += f[0].y, v[2] += f[0].z, v[3] += f[0].w;
        v[4] += f[32].x, v[5] += f[32].y, v[6] += f[32].z, v[7] += f[32].w;
    }
    put<MODE, T>(it, pr, 32 * tm + 16 * wave, 32 * tn, v, Eights{}, true, turn[wave]);
}

// Small matrices as a whole: X, its transpose and A (then B in its place) stay
// in the LDS of one workgroup through all steps, so that a call is one launch
// instead of three a step.
constexpr int kWholeWaves = 8;
constexpr int kWholeThreads = kWholeWaves * kWave;

struct WholeParams {
    int32_t steps;
    double scale;    // X_0's
    float keep;
    struct {
        float gram, poly, lin, diag, apply;   // as OrthParams has them
    } st[kWholeSteps];
};

// A plane in LDS: [part][row / 32][k / 8][row % 32][8], the 32 rows followed by
// 16 bytes that set the next k / 8 off by four banks.
struct LdsPlane {
    half8 *p;
    int rows, k8;   // blocks of 32 rows, of 8 k
    __device__ __forceinline__ int size() const { return rows * k8 * 33; }
    __device__ __forceinline__ half8 *at(int row, int k, int part) const
    {
        return p + part * size() + (row / 32 * k8 + k / 8) * 33 + row % 32;
    }
    // the operand of a matrix instruction: 16 rows, 32 k
    __device__ __forceinline__ half8 frag(int row, int k, int part, int lane) const
    {
        return *at(row + lane % 16, k + lane / 16 * 8, part);
    }
    // 4 consecutive k of a row
    __device__ __forceinline__ half4 *at4(int row, int k, int part) const
    {
        return reinterpret_cast<half4 *>(at(row, k, part)) + k / 4 % 2;
    }
    __device__ __forceinline__ _Float16 *at1(int row, int k, int part) const
    {
        return reinterpret_cast<_Float16 *>(at(row, k, part)) + k % 8;
    }
};

// 16 x 16 blocks of P Q^T (rows m of P, n of Q) over k in [0, K), K a multiple
// of 32: for each lane (n = lane % 16) rows m = 4 (lane / 16) .. + 3.
template <int BLOCKS>
__device__ __forceinline__ void block_products(const LdsPlane &P, const int (&m)[BLOCKS],
                                               const LdsPlane &Q, const int (&n)[BLOCKS], int K,
                                               int lane, floatx4 (&acc)[BLOCKS])
{
    floatx4 low[BLOCKS];   // (the small products')
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i)
        acc[i] = low[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < K; k += 32) {
        half8 p[BLOCKS][2], q[BLOCKS][2];
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                p[i][h] = P.frag(m[i], k, h, lane);
                q[i][h] = Q.frag(n[i], k, h, lane);
            }
#pragma unroll
        for (int t = 0; t < 3; ++t)
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                // (the large ones are added outside, where sums are rounded to
                // the nearest: the instruction's own lean towards zero)
                if (t)
                    low[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[i][t == 2], q[i][t == 1],
                                                                    low[i], 0, 0, 0);
                else
                    acc[i] += __builtin_amdgcn_mfma_f32_16x16x32_f16(
                        p[i][0], q[i][0], floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
            }
    }
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i)
        acc[i] += low[i];
}

template <bool UPDATE, class T>
__global__ __launch_bounds__(kWholeThreads) void k_orth_whole(OrthBatch b, WholeParams pr)
{
    // X and X^T of 64 x 256, A of 64 x 64
    __shared__ half8 lds[2 * 2 * (kWholeRows / 32) * (kWholeCols / 8) * 33 +
                         2 * (kWholeRows / 32) * (kWholeRows / 8) * 33];
    __shared__ double sums[kWholeWaves];
    const OrthItem &it = b.item[blockIdx.x];
    const int lane = threadIdx.x % kWave, wave = wave_id();
    const bool tall = it.rows > it.cols;
    constexpr int R = kWholeRows;
    const int C = it.ck;
    const LdsPlane X = {lds, R / 32, C / 8};
    const LdsPlane Xt = {lds + 2 * X.size(), C / 32, R / 8};
    const LdsPlane A = {Xt.p + 2 * Xt.size(), R / 32, R / 8};

    // U, eight consecutive elements of a row a thread, the rows side by side
    constexpr int N = kWholeRows * kWholeCols / 8 / kWholeThreads;
    const int ui = tall ? C : R, uk = (tall ? R : C) / 8;   // padded rows, eights of a row
    float u[N][8];
    double sum = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int q = threadIdx.x + j * kWholeThreads, i = q % ui, k = q / ui * 8;
        const int n = i < it.rows ? max(0, min(8, it.cols - k)) : 0;
        const auto x = load_some<T, 8>((const T *)it.u + (int64_t)i * it.ldu + k, n);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u[j][e] = (float)x[e];
            sum += (double)u[j][e] * (double)u[j][e];
        }
    }
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1)
        sum += __shfl_xor(sum, off);
    if (lane == 0)
        sums[wave] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < kWholeWaves; ++w)
        sum += sums[w];
    const double f = sum == 0 ? 0.0 : pr.scale / sqrt(sum);
    const LdsPlane P = tall ? Xt : X, Pt = tall ? X : Xt;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int q = threadIdx.x + j * kWholeThreads, i = q % ui, k = q / ui * 8;
        if (k >= 8 * uk)
            continue;
        half8 h, l;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = (float)((double)u[j][e] * f);
            h[e] = (_Float16)v;
            l[e] = (_Float16)(v - (float)h[e]);
        }
        *P.at(i, k, 0) = h;
        *P.at(i, k, 1) = l;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            *Pt.at1(k + e, i, 0) = h[e];
            *Pt.at1(k + e, i, 1) = l[e];
        }
    }
    __syncthreads();

    // 16 x 16 blocks: two of the 16 of A and B a wave, in one row of blocks
    // (all of them: a block is stored transposed, which is its mirror's place)
    const int am[2] = {wave / 2 * 16, wave / 2 * 16};
    const int an[2] = {wave % 2 * 32, wave % 2 * 32 + 16};
    const int lm = lane / 16 * 4, ln = lane % 16;
    auto split4 = [](const float (&v)[4], half4 &h, half4 &l) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h[e] = (_Float16)v[e];
            l[e] = (_Float16)(v[e] - (float)h[e]);
        }
    };
    for (int st = 0; st < pr.steps; ++st) {
        const auto p = pr.st[st];
        floatx4 acc[2];
        half4 h[2], l[2];
        // A = X X^T
        block_products<2>(X, am, X, an, C, lane, acc);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = acc[i][e] * p.gram;
            split4(v, h[i], l[i]);
            *A.at4(an[i] + ln, am[i] + lm, 0) = h[i];
            *A.at4(an[i] + ln, am[i] + lm, 1) = l[i];
        }
        __syncthreads();
        // B = a I + b A + c A A, over A once every wave has read it
        block_products<2>(A, am, A, an, R, lane, acc);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = fmaf((float)h[i][e] + (float)l[i][e], p.lin, acc[i][e] * p.poly) +
                       (am[i] + lm + e == an[i] + ln ? p.diag : 0.f);
            split4(v, h[i], l[i]);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            *A.at4(an[i] + ln, am[i] + lm, 0) = h[i];
            *A.at4(an[i] + ln, am[i] + lm, 1) = l[i];
        }
        __syncthreads();
        // X <- B X: two 16-wide columns of blocks of X a wave, over X once every
        // wave has read it
        floatx4 out[2][4];
        const int xm[4] = {0, 16, 32, 48};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int c = 16 * (wave + kWholeWaves * j), xn[4] = {c, c, c, c};
            if (c < C)
                block_products<4>(A, xm, Xt, xn, R, lane, out[j]);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int c = 16 * (wave + kWholeWaves * j) + ln;
            if (c - ln >= C)
                continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int m = 16 * i + lm;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = out[j][i][e] * p.apply;
                if (st + 1 < pr.steps) {
                    split4(v, h[0], l[0]);
                    *Xt.at4(c, m, 0) = h[0];
                    *Xt.at4(c, m, 1) = l[0];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        *X.at1(m + e, c, 0) = h[0][e];
                        *X.at1(m + e, c, 1) = l[0][e];
                    }
                    continue;
                }
                put_result<UPDATE, 4>(it, pr.keep, m, c, v, (T *)it.out);
            }
        }
        __syncthreads();
    }
}

// How the products of one kind run: the kernel, by its tile, and its
// workgroups.
struct OrthPlan {
    OrthParams pr;
    int32_t tile, blocks;   // 32 and 64: k_orth_small, 128 and 256: k_orth_gemm
    int32_t joins;          // split tiles, for k_orth_join
};

constexpr int kSlots = 256;    // CUs
constexpr int kMinChunk = 4;   // lines of a part, at least (an even number each)

// The fastest of the kernels by their times in us, as measured (MI355X, fp32
// 64 x 512 to 4,096 x 4,096; w is the lines, 32 k each, of one of the eight
// waves that share a small tile's k, n the workgroups of a round of 256):
//   32    3.9 + 0.7 w, or 2 + 3.2e-3 a tile + 4.2e-3 w a tile where that is more
//   64    1 + (4.5 + 1.65 w) for each 256 tiles
//   128   5.5 + (0.58 + 0.2 n / 256) a line of each round
//   256   8 + (2.0 + 0.6 n / 256) a line of each round
// A tile's k may be split where tiles are few or left over by whole rounds:
// the join takes 3.5 + 0.015 (128) or 4 + 0.045 (256) a part.  (1,024 x 4,096:
// X X^T 35 us with 64, 20 and 6 with 128 in seven parts each; B X 48 and 32;
// 256 x 256: 4.8 us with 32, 6.3 with 64, 11 to 13 with 128; 4,096 x 4,096:
// B X 418 with 128, 348 with 256.)  Past those sizes the times are the same
// lines carried on, and still choose: with the other tile of 128 and 256 for
// either symmetric product, or for B X, five steps take 2.5 and 10% longer for
// two 4,096 x 4,096 in one call (6,720 us), 2.7 and 7% for 5,120 x 5,120, 4.6
// and 12% for 8,192 x 8,192 (25,340).  Where the two are close they can err: 128
// for B X takes 1,285 us at 2,816 x 2,816, the 256 chosen 1,322.
template <int MODE>
OrthPlan plan_products(const OrthBatch &b)
{
    constexpr bool SYM = symmetric(MODE);
    OrthPlan best{};
    double time = 1e300;
    int32_t lines[kOrthItems], most = 0;
    for (int i = 0; i < b.n; ++i) {
        lines[i] = (MODE == kGram ? b.item[i].ck : b.item[i].rk) / kBlockK;
        most = std::max(most, lines[i]);
    }
    auto start = [&](int tile) {
        OrthPlan p{};
        p.tile = tile;
        for (int i = 0; i < b.n; ++i)
            p.pr.tile0[i + 1] = p.pr.tile0[i] + tiles_of(b.item[i], SYM, tile);
        for (int i = b.n + 1; i <= kOrthItems; ++i)
            p.pr.tile0[i] = INT32_MAX;
        p.blocks = p.pr.whole = p.pr.tile0[b.n];
        return p;
    };
    auto consider = [&](const OrthPlan &p, double t) {
        if (t < time) {
            time = t;
            best = p;
        }
    };
    auto shared = [](int n) { return (n + kSmallWaves - 1) / kSmallWaves; };
    {
        const OrthPlan p = start(32);
        double all = 0;
        for (int i = 0; i < b.n; ++i)
            all += (p.pr.tile0[i + 1] - p.pr.tile0[i]) * (3.2e-3 + 4.2e-3 * shared(lines[i]));
        consider(p, std::max(3.9 + 0.7 * shared(most), 2 + all));
    }
    {
        const OrthPlan p = start(64);
        consider(p, 1 + (p.blocks + kSlots - 1) / kSlots * (4.5 + 1.65 * shared(most)));
    }
    for (int tile = 128; tile <= 256; tile *= 2) {
        const OrthPlan all = start(tile);
        const int32_t tiles = all.blocks;
        const bool wide = tile == 256;
        // n workgroups of c lines each
        auto run = [&](int32_t n, int32_t c) {
            const double left = n % kSlots / (double)kSlots;
            return c * (wide ? n / kSlots * 2.6 + (left > 0 ? 2.0 + 0.6 * left : 0)
                             : n / kSlots * 0.78 + (left > 0 ? 0.58 + 0.2 * left : 0));
        };
        const double base = wide ? 8 : 5.5;
        consider(all, base + run(tiles, most));
        if (tiles % kSlots == 0)
            continue;
        // the tiles that whole rounds leave over, in `split` parts each
        for (int split = 2; split <= 16; split += split < 4 ? 1 : split / 4 * 2) {
            OrthPlan p = all;
            p.pr.whole = tiles - tiles % kSlots;
            p.pr.chunk = ((most + split - 1) / split + 1) / 2 * 2;
            if (p.pr.chunk < kMinChunk)
                break;
            p.joins = tiles - p.pr.whole;
            int32_t n = 0;
            for (int i = 0; i < b.n; ++i) {
                const int32_t left = p.pr.tile0[i + 1] - std::max(p.pr.whole, p.pr.tile0[i]);
                p.pr.parts[i] = (lines[i] + p.pr.chunk - 1) / p.pr.chunk;
                p.pr.work0[i] = p.pr.whole + n;
                n += std::max(0, left) * p.pr.parts[i];
            }
            for (int i = b.n; i < kOrthItems; ++i)
                p.pr.work0[i] = INT32_MAX;
            p.blocks = p.pr.whole + n;
            consider(p, base + run(p.pr.whole, most) + run(n, p.pr.chunk) +
                            (wide ? 4 + 0.045 * n : 3.5 + 0.015 * n));
        }
    }
    return best;
}

template <int MODE, class T, int TILE>
void gemm(const OrthBatch &b, const OrthPlan &p, hipStream_t s)
{
    constexpr int units = (TILE / 32) * (TILE / 32) * 2;   // waves that join a tile
    k_orth_gemm<MODE, T, TILE><<<p.blocks, Waves<TILE>::W * kWave, 0, s>>>(b, p.pr);
    if (p.joins > 0)
        k_orth_join<MODE, T, TILE>
            <<<p.joins * units / (kThreads / kWave), kThreads, 0, s>>>(b, p.pr);
}

// The product with X and the polynomial before it, together or one by one.
template <int MODE, class T>
hipError_t product(const OrthBatch &b, const OrthPlan &p, hipStream_t s);
template <int MODE, class T>
hipError_t poly_apply(const OrthBatch &b, const OrthPlan &poly, const OrthPlan &apply, bool fuse,
                      hipStream_t s)
{
    if (fuse) {
        k_orth_poly_apply<MODE, T>
            <<<apply.blocks, kFuseWaves * kWave, 0, s>>>(b, poly.pr, apply.pr);
        return hipGetLastError();
    }
    if (hipError_t e = product<kPoly, float>(b, poly, s))
        return e;
    return product<MODE, T>(b, apply, s);
}

template <int MODE, class T>
hipError_t product(const OrthBatch &b, const OrthPlan &p, hipStream_t s)
{
    switch (p.tile) {
    case 32:
        k_orth_small<MODE, T, 1, 4><<<p.blocks, kSmallWaves * kWave, 0, s>>>(b, p.pr);
        break;
    case 64:
        k_orth_small<MODE, T, 2, 2><<<p.blocks, kSmallWaves * kWave, 0, s>>>(b, p.pr);
        break;
    case 128: gemm<MODE, T, 128>(b, p, s); break;
    case 256: gemm<MODE, T, 256>(b, p, s); break;
    default: return hipErrorInvalidValue;
    }
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

constexpr int64_t kSplitFew = 1024;   // tiles

template <int THREADS>
hipError_t launch_split(const OrthBatch &b, int32_t type, dim3 grid, double scale, hipStream_t s)
{
    switch (type) {
    case kF32: k_orth_split<float, THREADS><<<grid, THREADS, 0, s>>>(b, scale); break;
    case kBF16: k_orth_split<__bf16, THREADS><<<grid, THREADS, 0, s>>>(b, scale); break;
    case kF16: k_orth_split<_Float16, THREADS><<<grid, THREADS, 0, s>>>(b, scale); break;
    default: return hipErrorInvalidValue;
    }
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
    // Few tiles are bound by latency, where twice the threads do half each:
    // the planes of a 100-256-256-47 network's matrices 5.9 us against 8.7, of
    // 1,024 x 4,096 (1,024 tiles) 12.2 against 14.7; of 4,096 x 4,096 39.6
    // against 38.0, of six matrices of 1,024 x 1,024 to 4,096 49 against 41.
    const bool few = (int64_t)gi * gj * b.n <= kSplitFew;
    return few ? launch_split<2 * kThreads>(b, type, dim3(gj, gi, b.n), std::ldexp(1.0, e), s)
               : launch_split<kThreads>(b, type, dim3(gj, gi, b.n), std::ldexp(1.0, e), s);
}

hipError_t launch_orth_whole(const OrthBatch &b, const OrthStep *st, int32_t steps, bool muon,
                             int32_t type, float keep, hipStream_t s)
{
    WholeParams pr{};
    pr.steps = steps;
    pr.keep = keep;
    pr.scale = std::ldexp(1.0, st[0].ex);
    for (int32_t k = 0; k < steps; ++k) {
        pr.st[k].gram = std::ldexp(1.f, st[k].ea - 2 * st[k].ex);
        pr.st[k].poly = std::ldexp(st[k].c, st[k].eb - 2 * st[k].ea);
        pr.st[k].lin = std::ldexp(st[k].b, st[k].eb - st[k].ea);
        pr.st[k].diag = std::ldexp(st[k].a, st[k].eb);
        pr.st[k].apply = std::ldexp(1.f, (k + 1 == steps ? 0 : st[k].en) - st[k].eb - st[k].ex);
    }
    if (muon) {
        k_orth_whole<true, float><<<b.n, kWholeThreads, 0, s>>>(b, pr);
        return hipGetLastError();
    }
    switch (type) {
    case kF32: k_orth_whole<false, float><<<b.n, kWholeThreads, 0, s>>>(b, pr); break;
    case kBF16: k_orth_whole<false, __bf16><<<b.n, kWholeThreads, 0, s>>>(b, pr); break;
    case kF16: k_orth_whole<false, _Float16><<<b.n, kWholeThreads, 0, s>>>(b, pr); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

size_t orth_partials(const OrthBatch &b)
{
    size_t most = 0;
    for (const OrthPlan &p :
         {plan_products<kGram>(b), plan_products<kPoly>(b), plan_products<kApply>(b)})
        most = std::max(most, (size_t)(p.blocks - p.pr.whole) * p.tile * p.tile * sizeof(float));
    return most;
}

hipError_t launch_orth_steps(const OrthBatch &b, const OrthStep *steps, int32_t n, bool muon,
                             int32_t type, float keep, float *partials, hipStream_t s)
{
    OrthPlan gram = plan_products<kGram>(b), poly = plan_products<kPoly>(b),
             apply = plan_products<kApply>(b);
    bool fuse = apply.tile == 32;
    for (int i = 0; i < b.n; ++i)
        fuse = fuse && b.item[i].rk <= kFuseRows;
    gram.pr.partials = poly.pr.partials = apply.pr.partials = partials;
    apply.pr.keep = keep;
    for (int32_t k = 0; k < n; ++k) {
        const OrthStep &st = steps[k];
        const bool last = k + 1 == n;
        gram.pr.alpha = std::ldexp(1.f, st.ea - 2 * st.ex);
        poly.pr.alpha = std::ldexp(st.c, st.eb - 2 * st.ea);
        poly.pr.lin = std::ldexp(st.b, st.eb - st.ea);
        poly.pr.diag = std::ldexp(st.a, st.eb);
        apply.pr.alpha = std::ldexp(1.f, (last ? 0 : st.en) - st.eb - st.ex);
        apply.pr.from = st.from;
        if (hipError_t e = product<kGram, float>(b, gram, s))
            return e;
        hipError_t e = hipErrorInvalidValue;
        if (!last)
            e = poly_apply<kApply, float>(b, poly, apply, fuse, s);
        else if (muon)
            e = poly_apply<kUpdate, float>(b, poly, apply, fuse, s);
        else if (type == kF32)
            e = poly_apply<kResult, float>(b, poly, apply, fuse, s);
        else if (type == kBF16)
            e = poly_apply<kResult, __bf16>(b, poly, apply, fuse, s);
        else if (type == kF16)
            e = poly_apply<kResult, _Float16>(b, poly, apply, fuse, s);
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace digest
