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

// The wave's number in its workgroup, in a scalar register.
__device__ __forceinline__ int wave_id()
{
    return __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
}

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
constexpr bool symmetric(int mode) { return mode == kGram || mode == kPoly; }

constexpr int kLine = 8;   // 16-byte chunks of a line

struct OrthParams {
    float alpha;         // plane products to the stored value's scale
    float diag, lin;     // kPoly: a 2^eb, b 2^(eb - ea)
    float keep;
    int32_t from;
    // Workgroups: the whole tiles [0, whole), then the parts of the others
    // (chunk lines of k each, item i's parts from work0[i] on).
    int32_t whole, chunk;
    int32_t tile0[kOrthItems + 1], work0[kOrthItems + 1], parts[kOrthItems];
    float *partials;
};

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

template <int MODE>
__device__ __forceinline__ void operands(const OrthItem &it, const OrthParams &pr, int &K,
                                         const char *&P, const char *&Q)
{
    K = MODE == kGram ? it.ck : it.rk;
    P = (const char *)(MODE == kGram ? it.X : MODE == kPoly ? it.A : it.B);
    Q = (const char *)(MODE == kGram ? it.X : MODE == kPoly ? it.A : it.Xt[pr.from]);
}

// Tile t of an item, tiles of BM x BN.  Symmetric products: the tiles that
// reach above the diagonal (BM = f BN), by column.
template <bool SYM, int BM, int BN>
__device__ __forceinline__ void tile_of(const OrthItem &it, int t, int &tm, int &tn)
{
    if constexpr (SYM) {
        constexpr int F = BM / BN;
        // columns F j .. F j + F - 1 have j + 1 tiles each: F j (j + 1) / 2 before them
        int j = (int)((sqrtf(8.f * (float)t / F + 1.f) - 1.f) * 0.5f);
        while (F * (j * (j + 1) / 2) > t)
            --j;
        while (F * ((j + 1) * (j + 2) / 2) <= t)
            ++j;
        t -= F * (j * (j + 1) / 2);
        tn = F * j + t / (j + 1);
        tm = t % (j + 1);
    } else {
        const int gm = (it.rp + BM - 1) / BM;
        tm = t % gm;
        tn = t / gm;
    }
}
template <bool SYM, int BM, int BN>
int tiles_of(const OrthItem &it)
{
    const int gm = (it.rp + BM - 1) / BM;
    if (!SYM)
        return gm * ((it.cp + BN - 1) / BN);
    constexpr int F = BM / BN;
    const int gn = (it.rp + BN - 1) / BN, j = gn / F;
    return F * (j * (j + 1) / 2) + (gn - F * j) * (j + 1);
}

// Stores four products of one column n, rows m .. m + 3 (a multiple of 4), of
// the 32 x 32 block at (mb, nb), which lies inside the padded product.
// `mirror`: the block's transposed is nobody else's to store.
template <int MODE, class T>
__device__ __forceinline__ void put(const OrthItem &it, const OrthParams &pr, int m, int n,
                                    const float (&x)[4], bool mirror)
{
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] = x[e] * pr.alpha;
    if constexpr (MODE == kPoly) {
        // (A is symmetric: its row n holds the four side by side)
        const _Float16 *a = (const _Float16 *)it.A + plane_at(n, it.rk, m);
        const half4 h = *reinterpret_cast<const half4 *>(a);
        const half4 l = *reinterpret_cast<const half4 *>(a + kBlockK);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = fmaf((float)h[e] + (float)l[e], pr.lin, v[e]) + (m + e == n ? pr.diag : 0.f);
    }
    if constexpr (MODE == kGram || MODE == kPoly || MODE == kApply) {
        half4 h, l;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h[e] = (_Float16)v[e];
            l[e] = (_Float16)(v[e] - (float)h[e]);
        }
        _Float16 *d = (_Float16 *)(MODE == kGram ? it.A : MODE == kPoly ? it.B : it.X);
        const int pitch = symmetric(MODE) ? it.rk : it.ck;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t at = plane_at(m + e, pitch, n);
            d[at] = h[e];
            d[at + kBlockK] = l[e];
        }
        if (mirror) {   // four consecutive k
            _Float16 *dt = symmetric(MODE) ? d : (_Float16 *)it.Xt[pr.from ^ 1];
            const int64_t at = plane_at(n, it.rk, m);
            *reinterpret_cast<half4 *>(dt + at) = h;
            *reinterpret_cast<half4 *>(dt + at + kBlockK) = l;
        }
    } else {
        const bool tall = it.rows > it.cols;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (m + e < it.r && n < it.c) {
                T *o = (T *)it.out + (tall ? (int64_t)n * it.ldo + m + e
                                           : (int64_t)(m + e) * it.ldo + n);
                if constexpr (MODE == kUpdate)
                    *o = (T)(pr.keep * (float)*o - it.scale * v[e]);
                else
                    *o = (T)v[e];
            }
    }
}

// A symmetric product's 32 x 32 block at (mb, nb): blocks below the diagonal
// are the mirror of those above.
template <int MODE>
__device__ __forceinline__ bool stored(const OrthItem &it, int mb, int nb)
{
    if (symmetric(MODE))
        return mb <= nb && nb < it.rk;
    return mb < it.rp && nb < it.cp;
}

// The large products: BM x BN of D per workgroup, WM x WN waves of TM x TN
// blocks of 32 x 32.  One line (32 k) of both operands' rows at a time in LDS,
// the next one on its way there.
template <int MODE, class T, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(WM *WN *kWave) void k_orth_gemm(OrthBatch b, OrthParams pr)
{
    constexpr int W = WM * WN, BM = WM * TM * 32, BN = WN * TN * 32;
    // [row][chunk]: chunk j of row i holds the line's chunk j ^ (i & 7), so
    // that eight rows' reads of one chunk fall into different banks
    __shared__ half8 lds0[(BM + BN) * kLine], lds1[(BM + BN) * kLine];

    int w = blockIdx.x, i = 0, t, part = -1;
    if (w < pr.whole) {
        w = (int)xcd_contiguous(w, pr.whole);
        while (i + 1 < b.n && w >= pr.tile0[i + 1])
            ++i;
        t = w - pr.tile0[i];
    } else {
        while (i + 1 < b.n && w >= pr.work0[i + 1])
            ++i;
        part = (w - pr.work0[i]) % pr.parts[i];
        t = max(pr.whole - pr.tile0[i], 0) + (w - pr.work0[i]) / pr.parts[i];
    }
    const OrthItem &it = b.item[i];
    int tm, tn, K;
    tile_of<symmetric(MODE), BM, BN>(it, t, tm, tn);
    const char *P, *Q;
    operands<MODE>(it, pr, K, P, Q);
    const int lane = threadIdx.x % kWave, wave = wave_id();
    const int wm = wave / WN * TM * 32, wn = wave % WN * TN * 32;

    floatx16 acc[TM][TN];
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                acc[x][y][e] = 0.f;

    // A wave's instruction takes 8 rows, 16 bytes a lane; rows past the
    // operand repeat its last eight (their products are not stored).
    const int64_t pitch = (int64_t)K * 4;   // bytes of a row
    const int prow = it.rp, qrow = symmetric(MODE) ? it.rp : it.cp;
    const int lrow = lane / kLine;
    const uint32_t loff = (uint32_t)(lrow * pitch) + 16 * ((lane % kLine) ^ lrow);
    auto load = [&](int kb, half8 *dst) {
#pragma unroll
        for (int q = 0; q < BM / 8; q += W) {
            const int row = 8 * (q + wave);
            const char *src = P + min(tm * BM + row, prow - 8) * pitch + kb * 128;
            __builtin_amdgcn_global_load_lds((global_void *)(src + loff),
                                             (lds_void *)(&dst[row * kLine]), 16, 0, 0);
        }
#pragma unroll
        for (int q = 0; q < BN / 8; q += W) {
            const int row = 8 * (q + wave);
            const char *src = Q + min(tn * BN + row, qrow - 8) * pitch + kb * 128;
            __builtin_amdgcn_global_load_lds((global_void *)(src + loff),
                                             (lds_void *)(&dst[(BM + row) * kLine]), 16, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto multiply = [&](const half8 *src) {
        const int r = lane % 32;
#pragma unroll
        for (int s = 0; s < kBlockK / 16; ++s) {
            half8 p[2][TM], q[2][TN];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int c = (4 * h + 2 * s + lane / 32) ^ (r & 7);
#pragma unroll
                for (int x = 0; x < TM; ++x)
                    p[h][x] = src[(wm + 32 * x + r) * kLine + c];
#pragma unroll
                for (int y = 0; y < TN; ++y)
                    q[h][y] = src[(BM + wn + 32 * y + r) * kLine + c];
            }
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll
                for (int x = 0; x < TM; ++x)
#pragma unroll
                    for (int y = 0; y < TN; ++y)
                        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                            p[k == 2][x], q[k == 1][y], acc[x][y], 0, 0, 0);
        }
    };
    const int k0 = part < 0 ? 0 : part * pr.chunk;
    const int k1 = part < 0 ? K / kBlockK : min(K / kBlockK, k0 + pr.chunk);
    load(k0, lds0);
    __syncthreads();
    for (int kb = k0; kb < k1; kb += 2) {   // (an even number of lines)
        load(kb + 1, lds1);
        multiply(lds0);
        __syncthreads();
        if (kb + 2 < k1)
            load(kb + 2, lds0);
        multiply(lds1);
        __syncthreads();
    }

    // (what the stores need is formed here, not kept through the loop)
    int lane_out = lane;
    asm volatile("" : "+v"(lane_out));
    // element e of a lane: row 8 (e / 4) + 4 (lane_out / 32) + e % 4, column lane % 32
    // of its 32 x 32 block
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y) {
            const int mb = tm * BM + wm + 32 * x, nb = tn * BN + wn + 32 * y;
            if (!stored<MODE>(it, mb, nb))
                continue;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = acc[x][y][4 * g + e];
                if (part < 0) {
                    put<MODE, T>(it, pr, mb + 8 * g + 4 * (lane_out / 32), nb + lane_out % 32, v,
                                 !symmetric(MODE) || mb != nb);
                } else {
                    float *d = pr.partials + (int64_t)(w - pr.whole) * (BM * BN) +
                               ((((wave * TM + x) * TN + y) * 4 + g) * kWave + lane_out) * 4;
                    *reinterpret_cast<float4 *>(d) = make_float4(v[0], v[1], v[2], v[3]);
                }
            }
        }
}

// Sums the parts of the tiles that were split, one wave a 32 x 32 block.
template <int MODE, class T, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(kThreads) void k_orth_join(OrthBatch b, OrthParams pr)
{
    constexpr int W = WM * WN, BM = WM * TM * 32, BN = WN * TN * 32, BLOCKS = W * TM * TN;
    const int lane = threadIdx.x % kWave;
    const int at = blockIdx.x * (kThreads / kWave) + wave_id();
    int tile = pr.whole + at / BLOCKS, i = 0;
    while (i + 1 < b.n && tile >= pr.tile0[i + 1])
        ++i;
    const OrthItem &it = b.item[i];
    const int first = max(pr.whole, pr.tile0[i]);   // the item's first split tile
    int tm, tn;
    tile_of<symmetric(MODE), BM, BN>(it, tile - pr.tile0[i], tm, tn);
    const int blk = at % BLOCKS, wave = blk / (TM * TN), x = blk / TN % TM, y = blk % TN;
    const int mb = tm * BM + (wave / WN * TM + x) * 32, nb = tn * BN + (wave % WN * TN + y) * 32;
    if (!stored<MODE>(it, mb, nb))
        return;
    const float *src = pr.partials +
                       (int64_t)(pr.work0[i] - pr.whole + (tile - first) * pr.parts[i]) * (BM * BN) +
                       (blk * 4 * kWave + lane) * 4;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < pr.parts[i]; ++p) {
            const float4 f = *reinterpret_cast<const float4 *>(src + (int64_t)p * (BM * BN) +
                                                               g * kWave * 4);
            v[0] += f.x, v[1] += f.y, v[2] += f.z, v[3] += f.w;
        }
        put<MODE, T>(it, pr, mb + 8 * g + 4 * (lane / 32), nb + lane % 32, v,
                     !symmetric(MODE) || mb != nb);
    }
}

// The small products, bound by latency: 64 x 64 of D per workgroup, whose
// waves split k among themselves (a line in turn, straight from memory into
// the registers that multiply) and add their sums through LDS in wave order.
constexpr int kSmallWaves = 8;
constexpr int kSmall = 64;

template <int MODE, class T>
__global__ __launch_bounds__(kSmallWaves *kWave) void k_orth_small(OrthBatch b, OrthParams pr)
{
    __shared__ float4 sum[kSmallWaves][16][kWave];
    int i = 0;
    const int w = (int)xcd_contiguous(blockIdx.x, gridDim.x);
    while (i + 1 < b.n && w >= pr.tile0[i + 1])
        ++i;
    const OrthItem &it = b.item[i];
    int tm, tn, K;
    tile_of<symmetric(MODE), kSmall, kSmall>(it, w - pr.tile0[i], tm, tn);
    const char *P, *Q;
    operands<MODE>(it, pr, K, P, Q);
    const int lane = threadIdx.x % kWave, wave = wave_id();
    const int64_t pitch = (int64_t)K * 4;
    const uint32_t loff = (uint32_t)((lane % 32) * pitch) + 16 * (lane / 32);
    P += tm * kSmall * pitch;
    Q += tn * kSmall * pitch;

    floatx16 acc[2][2];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                acc[x][y][e] = 0.f;
    struct Line {
        half8 p[2][2][2], q[2][2][2];   // [16 k][part][block]
    };
    auto load = [&](int kb, Line &l) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int64_t o = 32 * x * pitch + kb * 128 + 64 * h + 32 * s;
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
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int y = 0; y < 2; ++y)
                        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                            l.p[s][k == 2][x], l.q[s][k == 1][y], acc[x][y], 0, 0, 0);
    };
    const int nk = K / kBlockK;
    if (wave < nk) {
        Line l0, l1;
        load(wave, l0);
        for (int kb = wave; kb < nk; kb += 2 * kSmallWaves) {
            // (past the end: the last line again, not multiplied)
            load(min(kb + kSmallWaves, nk - 1), l1);
            multiply(l0);
            if (kb + kSmallWaves >= nk)
                break;
            load(min(kb + 2 * kSmallWaves, nk - 1), l0);
            multiply(l1);
        }
    }
    const int waves = min(kSmallWaves, nk);   // the others' sums are zero
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                sum[wave][(2 * x + y) * 4 + g][lane] =
                    make_float4(acc[x][y][4 * g], acc[x][y][4 * g + 1], acc[x][y][4 * g + 2],
                                acc[x][y][4 * g + 3]);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 16 / kSmallWaves; ++j) {
        const int at = wave * (16 / kSmallWaves) + j, x = at / 8, y = at / 4 % 2, g = at % 4;
        const int mb = tm * kSmall + 32 * x, nb = tn * kSmall + 32 * y;
        if (!stored<MODE>(it, mb, nb))
            continue;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < waves; ++p) {
            const float4 f = sum[p][at][lane];
            v[0] += f.x, v[1] += f.y, v[2] += f.z, v[3] += f.w;
        }
        put<MODE, T>(it, pr, mb + 8 * g + 4 * (lane / 32), nb + lane % 32, v,
                     !symmetric(MODE) || mb != nb);
    }
}

// The large kernel's shape, and its workgroups on the card at a time.
#ifndef ORTH_SHAPE
#define ORTH_SHAPE 2, 4, 4, 2
#endif
constexpr int kShape[4] = {ORTH_SHAPE};
constexpr int kBM = kShape[0] * kShape[2] * 32, kBN = kShape[1] * kShape[3] * 32;
#ifndef ORTH_SLOTS
#define ORTH_SLOTS 256
#endif
constexpr int kSlots = ORTH_SLOTS;
constexpr int kMinChunk = 4;   // lines of a part, at least (an even number each)

template <bool SYM>
int lines_of(const OrthItem &it, int mode)
{
    return (mode == kGram ? it.ck : it.rk) / kBlockK;
}

// Splits the k of the tiles that are left over when the whole ones have
// filled the card's slots evenly: into as many parts as there are slots.
template <int MODE>
int32_t plan_tiles(const OrthBatch &b, OrthParams &pr)
{
    constexpr bool SYM = symmetric(MODE);
    pr.tile0[0] = 0;
    for (int i = 0; i < b.n; ++i)
        pr.tile0[i + 1] = pr.tile0[i] + tiles_of<SYM, kBM, kBN>(b.item[i]);
    const int32_t tiles = pr.tile0[b.n];
    pr.whole = tiles - tiles % kSlots;
    auto parts = [&](int chunk) {
        int32_t n = 0;
        for (int i = 0; i < b.n; ++i) {
            const int left = pr.tile0[i + 1] - std::max(pr.whole, pr.tile0[i]);
            const int lines = lines_of<SYM>(b.item[i], MODE);
            pr.parts[i] = (lines + chunk - 1) / chunk;
            pr.work0[i] = pr.whole + n;
            if (left > 0)
                n += left * pr.parts[i];
        }
        pr.work0[b.n] = pr.whole + n;
        return n;
    };
    int most = 0;
    for (int i = 0; i < b.n; ++i)
        most = std::max(most, lines_of<SYM>(b.item[i], MODE));
    pr.chunk = kMinChunk;
    while (pr.chunk < most && parts(pr.chunk) > kSlots)
        pr.chunk += std::max(2, pr.chunk / 32 * 2);
    const int32_t n = parts(pr.chunk);
    if (n == tiles - pr.whole) {   // nothing to split
        pr.whole = tiles;
        return tiles;
    }
    return pr.whole + n;
}

// 64 x 64 tiles up to which the small kernel is the faster one.
constexpr int kSmallTiles = 512;
template <int MODE>
int32_t small_tiles(const OrthBatch &b, OrthParams &pr)
{
    pr.tile0[0] = 0;
    for (int i = 0; i < b.n; ++i)
        pr.tile0[i + 1] = pr.tile0[i] + tiles_of<symmetric(MODE), kSmall, kSmall>(b.item[i]);
    return pr.tile0[b.n];
}

template <int MODE, class T>
hipError_t gemm(const OrthBatch &b, OrthParams pr, hipStream_t s)
{
    int32_t n = small_tiles<MODE>(b, pr);
    if (n <= kSmallTiles) {
        k_orth_small<MODE, T><<<n, kSmallWaves * kWave, 0, s>>>(b, pr);
        return hipGetLastError();
    }
    n = plan_tiles<MODE>(b, pr);
    k_orth_gemm<MODE, T, ORTH_SHAPE><<<n, kShape[0] * kShape[1] * kWave, 0, s>>>(b, pr);
    if (pr.whole < pr.tile0[b.n])
        k_orth_join<MODE, T, ORTH_SHAPE>
            <<<(pr.tile0[b.n] - pr.whole) * (kBM / 32) * (kBN / 32) / (kThreads / kWave), kThreads, 0,
               s>>>(b, pr);
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

size_t orth_partials(const OrthBatch &b)
{
    OrthParams pr{};
    auto bytes = [&](int32_t small, int32_t work) {
        return small <= kSmallTiles ? 0 : (size_t)(work - pr.whole) * kBM * kBN * sizeof(float);
    };
    size_t most = 0;
    most = std::max(most, bytes(small_tiles<kGram>(b, pr), plan_tiles<kGram>(b, pr)));
    most = std::max(most, bytes(small_tiles<kPoly>(b, pr), plan_tiles<kPoly>(b, pr)));
    return std::max(most, bytes(small_tiles<kApply>(b, pr), plan_tiles<kApply>(b, pr)));
}

hipError_t launch_orth_step(const OrthBatch &b, const OrthStep &st, bool last, bool muon,
                            int32_t type, float keep, float *partials, hipStream_t s)
{
    OrthParams pr{};
    pr.partials = partials;
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
