// Orthogonalisation of matrices by Newton-Schulz products, and the weight update that uses it.
//     X_0 = U / max(|U|_F, eps), m <= n after a transposition;  A = X X^T;  P = a I + b A + c A A;  X <- P X
//     muon: M <- M + (1 - mu)(G - M), U = G + mu (M - G) or M;  W <- (1 - lr decay) W - lr sqrt(max(1, rows / cols)) X
//
// Arithmetic.  The products run on the 16-bit matrix cores: a float is the sum of two fp16 numbers, v = (h + l) / 4096, and
// v w = h h' + h l' + l h' with fp32 sums.  Two fp16 numbers hold 22 bits of it; the scale keeps what the second one drops at
// 2^-37 of a matrix whose largest value is 16, and the entries of X, A and P are bounded by their largest singular value,
// which the host bounds from the coefficients (below 16).  One fp16 number alone would leave an error of 2^-12 of X in every
// step, which later steps multiply by up to a: with a = 3.44 and five steps that is more than the rounding of a bf16 result.
//
// Memory.  X, X^T, A and P are kept in the order in which the matrix instruction reads its operand: blocks of 32 rows x 16
// columns, [lane][8 values] of the first numbers, then of the second ones, so that a staged tile is a run of whole kilobytes
// and a fragment is one conflict-free 16-byte read a lane.  Extents are padded to whole tiles with zeros, which stay zeros.
// X is needed with its columns along k (A) and with its rows along k (P X), so both orders are written.
//
// Launches cover all matrices of a call: a workgroup finds its matrix in the list of first tiles.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "launch.h"

namespace xc {

namespace {

constexpr float kOrthScale = 4096.f, kOrthUnscale = 1.f / (4096.f * 4096.f);
constexpr int kOrthItems = 24;      // matrices of one launch (as many as kernel arguments hold)
constexpr int kOrthTile = 64;       // extents are padded to this
constexpr int kOrthNorms = 64;      // most partial sums of a matrix' squares
constexpr int kBlockHalfs = 1024;   // 32 x 16 values, both numbers

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct OrthMat {
    const void *G;
    void *out;
    float *M;
    _Float16 *X, *Xt, *Xt2, *A, *P;     // fragment order
    float *A32;                         // [mp][mp]
    double *sq;                         // partial sums of squares
    int rows, cols, m, n, mp, np;       // m <= n
    int first[3];                       // first workgroup in launches over elements, tiles of A, tiles of X
    int nsq;
    float wscale;                       // lr sqrt(max(1, rows / cols))
};
struct OrthList {
    int count, g_dtype, out_dtype, muon, nesterov, steps;
    float a, b, c, eps, mu, keep;       // keep = 1 - lr decay
    OrthMat mat[kOrthItems];
};
static_assert(sizeof(OrthList) <= 4096, "kernel arguments");

__device__ inline const OrthMat &find_mat(const OrthList &L, int which, int &b)
{
    int i = 0;
    while (i + 1 < L.count && L.mat[i + 1].first[which] <= b) ++i;
    b -= L.mat[i].first[which];
    return L.mat[i];
}

__device__ inline float orth_get(const void *p, int dtype, size_t i)
{
    if (dtype == XCONV_F32) return static_cast<const float *>(p)[i];
    const uint16_t h = static_cast<const uint16_t *>(p)[i];
    return dtype == XCONV_BF16 ? bf16_to_f32(h) : f16_to_f32(h);
}
__device__ inline void orth_put(void *p, int dtype, size_t i, float v)
{
    if (dtype == XCONV_F32) static_cast<float *>(p)[i] = v;
    else static_cast<uint16_t *>(p)[i] = dtype == XCONV_BF16 ? f32_to_bf16_rne(v) : f32_to_f16_rne(v);
}
__device__ inline float update_of(float g, float m, const OrthList &L) { return L.nesterov ? g + L.mu * (m - g) : m; }

// eight values as two fp16 numbers each, stored at their place (row r, columns k .. k + 7) of a matrix in fragment order
__device__ inline void put_pieces(_Float16 *frag, int r, int k, int kblocks, const float (&v)[8])
{
    h8 h, l;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = v[i] * kOrthScale;
        h[i] = (_Float16)s;
        l[i] = (_Float16)(s - (float)h[i]);
    }
    _Float16 *p = frag + ((size_t)(r >> 5) * kblocks + (k >> 4)) * kBlockHalfs + ((r & 31) + 32 * ((k >> 3) & 1)) * 8;
    *reinterpret_cast<h8 *>(p) = h;
    *reinterpret_cast<h8 *>(p + 512) = l;
}

// ---- momentum and the sum of squares -------------------------------------------------------------------------------
__global__ __launch_bounds__(kThreads) void orth_norm_kernel(OrthList L)
{
    __shared__ double red[kThreads / 64];
    int b = blockIdx.x;
    const OrthMat &q = find_mat(L, 0, b);
    const size_t n = (size_t)q.rows * q.cols, step = (size_t)q.nsq * kThreads;
    double s = 0.0;
    for (size_t i = (size_t)b * kThreads + threadIdx.x; i < n; i += step) {
        float u = orth_get(q.G, L.g_dtype, i);
        if (L.muon) {
            float m = q.M[i];
            m = m + (u - m) * (1.f - L.mu);
            q.M[i] = m;
            u = update_of(u, m, L);
        }
        s += (double)u * u;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) q.sq[b] = (red[0] + red[1]) + (red[2] + red[3]);
}

// ---- X_0 in both orders: a workgroup takes 64 x 64 values ----------------------------------------------------------
// t[r][c]: r along m, c along n
__device__ inline void emit_x(const float (*t)[kOrthTile + 1], const OrthMat &q, _Float16 *xt, int m0, int n0)
{
    for (int u = threadIdx.x; u < 512; u += kThreads) {
        const int r = u & 63, c = (u >> 6) * 8;
        float v[8], w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = t[r][c + i];
            w[i] = t[c + i][r];
        }
        put_pieces(q.X, m0 + r, n0 + c, q.np / 16, v);
        put_pieces(xt, n0 + r, m0 + c, q.mp / 16, w);
    }
}

__global__ __launch_bounds__(kThreads) void orth_start_kernel(OrthList L)
{
    __shared__ float t[kOrthTile][kOrthTile + 1];
    int b = blockIdx.x;
    const OrthMat &q = find_mat(L, 2, b);
    const int tm = q.mp / kOrthTile, m0 = (b % tm) * kOrthTile, n0 = (b / tm) * kOrthTile;
    double s = 0.0;
    for (int i = 0; i < q.nsq; ++i) s += q.sq[i];
    const double norm = sqrt(s), d = norm < (double)L.eps ? (double)L.eps : norm;      // (a NaN stays one)
    const double inv = d == 0.0 ? 0.0 : 1.0 / d;                                      // (eps = 0 and a zero matrix)
    const bool tall = q.rows > q.cols;
    const int r0 = tall ? n0 : m0, c0 = tall ? m0 : n0;
    for (int u = threadIdx.x; u < kOrthTile * kOrthTile; u += kThreads) {
        const int r = u / kOrthTile, c = u % kOrthTile;
        float v = 0.f;
        if (r0 + r < q.rows && c0 + c < q.cols) {
            const size_t i = (size_t)(r0 + r) * q.cols + c0 + c;
            v = orth_get(q.G, L.g_dtype, i);
            if (L.muon) v = update_of(v, q.M[i], L);
            v = (float)((double)v * inv);
        }
        if (tall) t[c][r] = v;
        else t[r][c] = v;
    }
    __syncthreads();
    emit_x(t, q, q.Xt, m0, n0);
}

// ---- products ------------------------------------------------------------------------------------------------------
// c[64 x 64] = sum over kb in [kb0, kb1) of rows ra .. of Fa times rows rb .. of Fb (both in fragment order with kblocks
// blocks a row of blocks); wave w computes rows 32 (w / 2), columns 32 (w % 2)
constexpr int kKS = 4;     // blocks of 16 a step

__device__ inline void tile_product(f32x16 &acc, const _Float16 *Fa, int ra, const _Float16 *Fb, int rb, int kblocks, int kb0, int kb1, uint4 *lds)
{
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int wa = wave >> 1, wb = wave & 1;
    // units of 16 bytes: a side is 2 row blocks of kKS blocks of 128 units
    constexpr int kSide = 2 * kKS * 128, kPer = 2 * kSide / kThreads;
    for (int kb = kb0; kb < kb1; kb += kKS) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int u = j * kThreads + tid, side = u / kSide, v = u % kSide, blk = v / (kKS * 128), off = v % (kKS * 128);   // kb1 - kb0 is whole steps
            const _Float16 *F = side ? Fb : Fa;
            const int row = (side ? rb : ra) / 32 + blk;
            const uint4 *src = reinterpret_cast<const uint4 *>(F + ((size_t)row * kblocks + kb) * kBlockHalfs) + off;
            lds[u] = *src;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kKS; ++k) {
            const uint4 *pa = lds + (wa * kKS + k) * 128 + lane, *pb = lds + kSide + (wb * kKS + k) * 128 + lane;
            const h8 ah = __builtin_bit_cast(h8, pa[0]), al = __builtin_bit_cast(h8, pa[64]);
            const h8 bh = __builtin_bit_cast(h8, pb[0]), bl = __builtin_bit_cast(h8, pb[64]);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, bh, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bl, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bh, acc, 0, 0, 0);
        }
    }
}
// the accumulators, in true scale, as t[row][column]
__device__ inline void tile_to_lds(const f32x16 &acc, float (*t)[kOrthTile + 1])
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) t[32 * (wave >> 1) + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3)][32 * (wave & 1) + (lane & 31)] = acc[i] * kOrthUnscale;
    __syncthreads();
}

union OrthLds {
    uint4 stage[2 * 2 * kKS * 128];
    float t[kOrthTile][kOrthTile + 1];
};

// pair (i <= j) of tiles of a symmetric matrix with T rows of tiles
__device__ inline void pair_of(int b, int &i, int &j)
{
    j = (int)((sqrtf(8.f * (float)b + 1.f) - 1.f) * 0.5f);
    while ((j + 1) * (j + 2) / 2 <= b) ++j;
    while (j * (j + 1) / 2 > b) --j;
    i = b - j * (j + 1) / 2;
}

// POLY 0: A = X X^T, also as plain floats.  1: P = a I + b A + c A A
template <int POLY> __global__ __launch_bounds__(kThreads) void orth_square_kernel(OrthList L)
{
    __shared__ OrthLds lds;
    int b = blockIdx.x;
    const OrthMat &q = find_mat(L, 1, b);
    int ti, tj;
    pair_of(b, ti, tj);
    const int i0 = ti * kOrthTile, j0 = tj * kOrthTile;
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    const int kblocks = (POLY ? q.mp : q.np) / 16;
    const _Float16 *F = POLY ? q.A : q.X;
    tile_product(acc, F, i0, F, j0, kblocks, 0, kblocks, lds.stage);
    tile_to_lds(acc, lds.t);
    _Float16 *out = POLY ? q.P : q.A;
    if constexpr (POLY == 1) {
        for (int u = threadIdx.x; u < kOrthTile * kOrthTile; u += kThreads) {
            const int r = u / kOrthTile, c = u % kOrthTile;
            float v = L.b * q.A32[(size_t)(i0 + r) * q.mp + j0 + c] + L.c * lds.t[r][c];
            if (i0 + r == j0 + c && i0 + r < q.m) v += L.a;
            lds.t[r][c] = v;
        }
    } else {
        for (int u = threadIdx.x; u < kOrthTile * kOrthTile; u += kThreads) {
            const int r = u / kOrthTile, c = u % kOrthTile;
            q.A32[(size_t)(i0 + r) * q.mp + j0 + c] = lds.t[r][c];
        }
    }
    __syncthreads();
    for (int u = threadIdx.x; u < 512; u += kThreads) {
        const int r = u & 63, c = (u >> 6) * 8;
        float v[8], w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = lds.t[r][c + i];
            w[i] = lds.t[c + i][r];
        }
        put_pieces(out, i0 + r, j0 + c, q.mp / 16, v);
        if (ti != tj) put_pieces(out, j0 + r, i0 + c, q.mp / 16, w);
    }
}

// the result of the last step, or X_0 when there is no step: O, or the update of W
__device__ inline void finish(const float (*t)[kOrthTile + 1], const OrthMat &q, const OrthList &L, int m0, int n0)
{
    const bool tall = q.rows > q.cols;
    const int r0 = tall ? n0 : m0, c0 = tall ? m0 : n0;
    for (int u = threadIdx.x; u < kOrthTile * kOrthTile; u += kThreads) {
        const int r = u / kOrthTile, c = u % kOrthTile;
        if (r0 + r >= q.rows || c0 + c >= q.cols) continue;
        const size_t i = (size_t)(r0 + r) * q.cols + c0 + c;
        float v = tall ? t[c][r] : t[r][c];
        if (L.muon) v = orth_get(q.out, L.out_dtype, i) * L.keep - q.wscale * v;
        orth_put(q.out, L.out_dtype, i, v);
    }
}

// X <- P X, from the transposed X `from` to X and `to`; last: to the result instead
__global__ __launch_bounds__(kThreads) void orth_apply_kernel(OrthList L, int odd, int last)
{
    __shared__ OrthLds lds;
    int b = blockIdx.x;
    const OrthMat &q = find_mat(L, 2, b);
    const int tm = q.mp / kOrthTile, m0 = (b % tm) * kOrthTile, n0 = (b / tm) * kOrthTile;
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    const int kblocks = q.mp / 16;
    tile_product(acc, q.P, m0, odd ? q.Xt2 : q.Xt, n0, kblocks, 0, kblocks, lds.stage);
    tile_to_lds(acc, lds.t);
    if (last) finish(lds.t, q, L, m0, n0);
    else emit_x(lds.t, q, odd ? q.Xt : q.Xt2, m0, n0);
}

// no steps: X_0 is the result
__global__ __launch_bounds__(kThreads) void orth_none_kernel(OrthList L)
{
    __shared__ float t[kOrthTile][kOrthTile + 1];
    int b = blockIdx.x;
    const OrthMat &q = find_mat(L, 2, b);
    const int tm = q.mp / kOrthTile, m0 = (b % tm) * kOrthTile, n0 = (b / tm) * kOrthTile;
    for (int u = threadIdx.x; u < 64 * 64; u += kThreads) {
        const int r = u / 64, c = u % 64, row = n0 + c, k = m0 + r;
        const _Float16 *p = q.Xt + ((size_t)(row >> 5) * (q.mp / 16) + (k >> 4)) * kBlockHalfs + ((row & 31) + 32 * ((k >> 3) & 1)) * 8 + (k & 7);
        t[r][c] = ((float)p[0] + (float)p[512]) / kOrthScale;
    }
    __syncthreads();
    finish(t, q, L, m0, n0);
}

// ---- host ----------------------------------------------------------------------------------------------------------
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

struct OrthSizes {
    int m, n, mp, np;
    size_t x, a;      // bytes of a matrix in fragment order
};
OrthSizes sizes_of(const xconv_orth_item &it)
{
    OrthSizes s;
    s.m = std::min(it.rows, it.cols);
    s.n = std::max(it.rows, it.cols);
    s.mp = round_up(s.m, kOrthTile);
    s.np = round_up(s.n, kOrthTile);
    s.x = up256((size_t)s.mp * s.np * 4);
    s.a = up256((size_t)s.mp * s.mp * 4);
    return s;
}
size_t item_bytes(const xconv_orth_item &it)
{
    const OrthSizes s = sizes_of(it);
    return 3 * s.x + 3 * s.a + up256(kOrthNorms * sizeof(double));
}

}  // namespace

// the matrices go through in runs of kOrthItems, one run after the other through the same scratch
size_t orth_ws_bytes(const xconv_orth_item *items, int count)
{
    size_t most = 256;
    for (int at = 0; at < count; at += kOrthItems) {
        size_t sum = 0;
        for (int i = at; i < std::min(count, at + kOrthItems); ++i) sum += item_bytes(items[i]);
        most = std::max(most, sum);
    }
    return most;
}

hipError_t launch_orth(const xconv_orth_item *items, int count, const xconv_orth_args *args, const xconv_muon_args *muon, void *ws, hipStream_t st)
{
    for (int at = 0; at < count; at += kOrthItems) {
        OrthList L{};
        L.count = std::min(kOrthItems, count - at);
        L.g_dtype = args->g_dtype; L.out_dtype = args->out_dtype; L.steps = args->steps;
        L.a = args->a; L.b = args->b; L.c = args->c; L.eps = args->eps;
        if (muon) {
            L.muon = 1; L.nesterov = muon->nesterov != 0; L.mu = muon->momentum;
            L.keep = (float)(1.0 - (double)muon->lr * muon->weight_decay);
        }
        char *p = static_cast<char *>(ws);
        auto take = [&](size_t bytes) { char *r = p; p += bytes; return r; };
        int total[3] = {0, 0, 0};
        for (int i = 0; i < L.count; ++i) {
            const xconv_orth_item &it = items[at + i];
            const OrthSizes s = sizes_of(it);
            OrthMat &q = L.mat[i];
            q.G = it.G_dev; q.out = it.out_dev; q.M = it.M_dev;
            q.rows = it.rows; q.cols = it.cols; q.m = s.m; q.n = s.n; q.mp = s.mp; q.np = s.np;
            q.X = (_Float16 *)take(s.x); q.Xt = (_Float16 *)take(s.x); q.Xt2 = (_Float16 *)take(s.x);
            q.A = (_Float16 *)take(s.a); q.P = (_Float16 *)take(s.a); q.A32 = (float *)take(s.a);
            q.sq = (double *)take(up256(kOrthNorms * sizeof(double)));
            q.nsq = (int)std::min<size_t>(kOrthNorms, ((size_t)it.rows * it.cols + 4095) / 4096);
            if (muon) q.wscale = (float)((double)muon->lr * std::sqrt(std::max(1.0, (double)it.rows / it.cols)));
            const int tm = s.mp / kOrthTile, tn = s.np / kOrthTile;
            const int blocks[3] = {q.nsq, tm * (tm + 1) / 2, tm * tn};
            for (int k = 0; k < 3; ++k) {
                q.first[k] = total[k];
                total[k] += blocks[k];
            }
        }
        const dim3 block(kThreads);
        hipLaunchKernelGGL(orth_norm_kernel, dim3(total[0]), block, 0, st, L);
        hipLaunchKernelGGL(orth_start_kernel, dim3(total[2]), block, 0, st, L);
        if (args->steps == 0) hipLaunchKernelGGL(orth_none_kernel, dim3(total[2]), block, 0, st, L);
        for (int k = 0; k < args->steps; ++k) {
            hipLaunchKernelGGL(orth_square_kernel<0>, dim3(total[1]), block, 0, st, L);
            hipLaunchKernelGGL(orth_square_kernel<1>, dim3(total[1]), block, 0, st, L);
            hipLaunchKernelGGL(orth_apply_kernel, dim3(total[2]), block, 0, st, L, k & 1, k + 1 == args->steps);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace xc
