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
constexpr int kOrthItems = 20;      // matrices of one launch (as many as kernel arguments hold)
constexpr int kOrthTile = 64;       // extents are padded to this or twice this
constexpr int kOrthNorms = 512;     // most partial sums of a matrix' squares
constexpr int kBlockHalfs = 1024;   // 32 x 16 values, both numbers

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct OrthMat {
    const void *G;
    void *out;
    float *M;
    _Float16 *X, *Xt, *Xt2, *A, *P;     // fragment order
    float *A32;                         // [mp][mp]
    double *sq;                         // partial sums of squares
    float *part;                        // partial products of X X^T, [tile][split][tile values]
    int rows, cols, m, n, mp, np;       // m <= n
    int first[4];                       // first workgroup in launches over elements, tiles of A, tiles of X, 64 x 64 tiles of X
    int nsq;
    int big;                            // tiles of 128 x 128 (else 64 x 64)
    int splits, kbs;                    // X X^T: runs of kbs blocks of 16 columns
    int gfirst, jfirst;                 // first workgroup in the launch of X X^T and of the one that joins it
    float wscale;                       // lr sqrt(max(1, rows / cols))
};
struct OrthScalars {
    int count, g_dtype, out_dtype, muon, nesterov;
    float a, b, c, eps, mu, keep;       // keep = 1 - lr decay
};
struct OrthList {
    OrthScalars s;
    OrthMat mat[kOrthItems];
};
static_assert(sizeof(OrthList) <= 4096, "kernel arguments");
// What the launches after the first are given: the list lies in the scratch
struct OrthRef {
    OrthScalars s;
    const OrthMat *mat;
};

// the matrix of workgroup b in a launch whose first workgroups are `first`; b becomes the workgroup's number in the matrix
template <class F> __device__ inline const OrthMat &find_mat(const OrthMat *mat, int count, F &&first, int &b)
{
    int lo = 0, hi = count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first(mat[mid]) <= b) lo = mid;
        else hi = mid - 1;
    }
    b -= first(mat[lo]);
    return mat[lo];
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
__device__ inline float update_of(float g, float m, const OrthScalars &L) { return L.nesterov ? g + L.mu * (m - g) : m; }

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

// four values from element i on, at the alignment of an element
struct __attribute__((packed, aligned(4))) Loose4 { uint32_t w[4]; };
struct __attribute__((packed, aligned(2))) Loose2 { uint32_t w[2]; };
__device__ inline void orth_get4(const void *p, int dtype, size_t i, float (&v)[4])
{
    if (dtype == XCONV_F32) {
        const Loose4 t = *reinterpret_cast<const Loose4 *>(static_cast<const float *>(p) + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(t.w[k]);
    } else {
        const Loose2 t = *reinterpret_cast<const Loose2 *>(static_cast<const uint16_t *>(p) + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint16_t h = (uint16_t)(t.w[k >> 1] >> (16 * (k & 1)));
            v[k] = dtype == XCONV_BF16 ? bf16_to_f32(h) : f16_to_f32(h);
        }
    }
}

// ---- momentum and the sum of squares; the list of matrices goes to the scratch ------------------------------------
__global__ __launch_bounds__(kThreads) void orth_norm_kernel(OrthList L, OrthMat *list)
{
    __shared__ double red[kThreads / 64];
    int b = blockIdx.x;
    if (b == 0) {
        const uint32_t *from = reinterpret_cast<const uint32_t *>(L.mat);
        uint32_t *to = reinterpret_cast<uint32_t *>(list);
        for (int i = threadIdx.x; i < (int)(L.s.count * sizeof(OrthMat) / 4); i += kThreads) to[i] = from[i];
    }
    const OrthMat &q = find_mat(L.mat, L.s.count, [](const OrthMat &m) { return m.first[0]; }, b);
    const size_t n = (size_t)q.rows * q.cols, step = (size_t)q.nsq * kThreads * 4;
    double s = 0.0;
    for (size_t i = ((size_t)b * kThreads + threadIdx.x) * 4; i < n; i += step) {
        float u[4], m[4];
        const int k1 = n - i < 4 ? (int)(n - i) : 4;
        if (k1 == 4) {
            orth_get4(q.G, L.s.g_dtype, i, u);
            if (L.s.muon) orth_get4(q.M, XCONV_F32, i, m);
        } else {
            for (int k = 0; k < 4; ++k) {
                u[k] = k < k1 ? orth_get(q.G, L.s.g_dtype, i + k) : 0.f;
                m[k] = L.s.muon && k < k1 ? q.M[i + k] : 0.f;
            }
        }
        if (L.s.muon) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                m[k] = m[k] + (u[k] - m[k]) * (1.f - L.s.mu);
                u[k] = update_of(u[k], m[k], L.s);
            }
            if (k1 == 4) {
                *reinterpret_cast<Loose4 *>(q.M + i) = Loose4{{__float_as_uint(m[0]), __float_as_uint(m[1]), __float_as_uint(m[2]), __float_as_uint(m[3])}};
            } else {
                for (int k = 0; k < k1; ++k) q.M[i + k] = m[k];
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) s += (double)u[k] * u[k];
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) q.sq[b] = (red[0] + red[1]) + (red[2] + red[3]);
}
// the sum of a matrix' partial sums, in order, for every thread of the workgroup
__device__ inline double sum_squares(const OrthMat &q)
{
    __shared__ double red[kThreads / 64];
    double s = 0.0;
    for (int i = threadIdx.x; i < q.nsq; i += kThreads) s += q.sq[i];
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// ---- X_0 in both orders: a workgroup takes 64 x 64 values ----------------------------------------------------------
// t[r][c], r < TM along m, c < TN along n, in both orders
template <int TM, int TN> __device__ inline void emit_x(const float (*t)[TN + 1], const OrthMat &q, _Float16 *xt, int m0, int n0)
{
    for (int u = threadIdx.x; u < TM * TN / 8; u += kThreads) {
        float v[8];
        int r = u % TM, c = u / TM * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = t[r][c + i];
        put_pieces(q.X, m0 + r, n0 + c, q.np / 16, v);
        r = u / TN * 8;
        c = u % TN;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = t[r + i][c];
        put_pieces(xt, n0 + c, m0 + r, q.mp / 16, v);
    }
}
// the part of tile b (of tm tiles along m)
struct TileAt {
    int m0, n0;
};
template <int TM, int TN> __device__ inline TileAt tile_at(const OrthMat &q, int b)
{
    const int tm = q.mp / TM;
    return {(b % tm) * TM, (b / tm) * TN};
}

__global__ __launch_bounds__(kThreads) void orth_start_kernel(OrthRef L)
{
    __shared__ float t[kOrthTile][kOrthTile + 1];
    int b = blockIdx.x;
    const OrthMat &q = find_mat(L.mat, L.s.count, [](const OrthMat &m) { return m.first[3]; }, b);
    const TileAt at = tile_at<kOrthTile, kOrthTile>(q, b);
    const double norm = sqrt(sum_squares(q)), d = norm < (double)L.s.eps ? (double)L.s.eps : norm;      // (a NaN stays one)
    const double inv = d == 0.0 ? 0.0 : 1.0 / d;                                                         // (eps = 0 and a zero matrix)
    const bool tall = q.rows > q.cols;
    const int r0 = tall ? at.n0 : at.m0, c0 = tall ? at.m0 : at.n0;
    constexpr int kRound = 4;
#pragma unroll
    for (int j = 0; j < kOrthTile * kOrthTile / kThreads; j += kRound) {
        float v[kRound], m[kRound];
#pragma unroll
        for (int k = 0; k < kRound; ++k) {
            const int u = (j + k) * kThreads + threadIdx.x, r = r0 + u / kOrthTile, c = c0 + u % kOrthTile;
            const bool on = r < q.rows && c < q.cols;
            const size_t i = (size_t)r * q.cols + c;
            v[k] = on ? orth_get(q.G, L.s.g_dtype, i) : 0.f;
            m[k] = on && L.s.muon ? q.M[i] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < kRound; ++k) {
            const int u = (j + k) * kThreads + threadIdx.x, r = u / kOrthTile, c = u % kOrthTile;
            if (L.s.muon) v[k] = update_of(v[k], m[k], L.s);
            const float x = r0 + r < q.rows && c0 + c < q.cols ? (float)((double)v[k] * inv) : 0.f;
            if (tall) t[c][r] = x;
            else t[r][c] = x;
        }
    }
    __syncthreads();
    emit_x<kOrthTile, kOrthTile>(t, q, q.Xt, at.m0, at.n0);
}

// ---- products ------------------------------------------------------------------------------------------------------
// A workgroup's tile: 64 MT rows of one matrix times 64 NT rows of another (rows along k, fragment order with kblocks blocks a
// row of blocks), blocks kb0 .. kb1 - 1; wave w computes rows 32 MT (w / 2), columns 32 NT (w % 2).  Steps of KS blocks are
// staged through registers into one of two buffers while the other one is used: one barrier a step.
constexpr int kStageUnits = 2048;     // 16-byte units of a step, 8 a thread
template <int MT, int NT> struct Tile {
    static constexpr int TM = 64 * MT, TN = 64 * NT, KS = kStageUnits / (2 * (MT + NT) * 128);
    f32x16 acc[MT][NT];

    __device__ void clear()
    {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    }
    static constexpr int kRun = KS * 128, kPer = kStageUnits / kThreads;
    __device__ static void load(u32x4 (&r)[kPer], const _Float16 *Fa, int ra, const _Float16 *Fb, int rb, int kblocks, int kb)
    {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            // (a run is a whole number of rounds of the workgroup, or half of one)
            const int blk = j * kThreads / kRun, off = (j * kThreads) % kRun + (int)threadIdx.x;
            const bool second = blk >= 2 * MT;
            const int row = second ? rb / 32 + blk - 2 * MT : ra / 32 + blk;
            r[j] = reinterpret_cast<const u32x4 *>((second ? Fb : Fa) + ((size_t)row * kblocks + kb) * kBlockHalfs)[off];
        }
    }
    __device__ static void store(const u32x4 (&r)[kPer], u32x4 *lds)
    {
#pragma unroll
        for (int j = 0; j < kPer; ++j) lds[j * kThreads + threadIdx.x] = r[j];
    }
    __device__ void multiply(const u32x4 *lds)
    {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wa = wave >> 1, wb = wave & 1;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            h8 a[2][MT], b[2][NT];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
#pragma unroll
                for (int i = 0; i < MT; ++i) a[p][i] = __builtin_bit_cast(h8, lds[((wa * MT + i) * KS + k) * 128 + p * 64 + lane]);
#pragma unroll
                for (int j = 0; j < NT; ++j) b[p][j] = __builtin_bit_cast(h8, lds[((2 * MT + wb * NT + j) * KS + k) * 128 + p * 64 + lane]);
            }
            // the small products first
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[p == 0][i], b[p == 1][j], acc[i][j], 0, 0, 0);
        }
    }
    // lds: two stages
    __device__ void product(const _Float16 *Fa, int ra, const _Float16 *Fb, int rb, int kblocks, int kb0, int kb1, u32x4 *lds)
    {
        clear();
        u32x4 r[kPer];
        load(r, Fa, ra, Fb, rb, kblocks, kb0);
        store(r, lds);
        __syncthreads();
        int at = 0;
        for (int kb = kb0 + KS; kb < kb1; kb += KS) {
            load(r, Fa, ra, Fb, rb, kblocks, kb);
            multiply(lds + at * kStageUnits);
            at ^= 1;
            store(r, lds + at * kStageUnits);
            __syncthreads();
        }
        multiply(lds + at * kStageUnits);
        __syncthreads();
    }
    // the sums, in true scale, as t[row][column]
    __device__ void spread(float (*t)[TN + 1]) const
    {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    t[32 * (MT * (wave >> 1) + i) + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)][32 * (NT * (wave & 1) + j) + (lane & 31)] = acc[i][j][e] * kOrthUnscale;
        __syncthreads();
    }
    // partial sums, in the order of the registers
    __device__ void put_part(float *part) const
    {
        f32x4 *p = reinterpret_cast<f32x4 *>(part) + threadIdx.x;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    p[((i * NT + j) * 4 + e) * kThreads] = f32x4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
    }
    __device__ void add_part(const float *part)
    {
        const f32x4 *p = reinterpret_cast<const f32x4 *>(part) + threadIdx.x;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x4 v = p[((i * NT + j) * 4 + e) * kThreads];
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[i][j][4 * e + k] += v[k];
                }
    }
};

union OrthLds {
    u32x4 stage[2 * kStageUnits];
    float small[64][64 + 1];
    float large[128][128 + 1];
};
template <int T> __device__ inline float (*tile_of(OrthLds &l))[T + 1]
{
    if constexpr (T == 64) return l.small;
    else return l.large;
}

// pair (i <= j) of tiles of a symmetric matrix with T rows of tiles
__device__ inline void pair_of(int b, int &i, int &j)
{
    j = (int)((sqrtf(8.f * (float)b + 1.f) - 1.f) * 0.5f);
    while ((j + 1) * (j + 2) / 2 <= b) ++j;
    while (j * (j + 1) / 2 > b) --j;
    i = b - j * (j + 1) / 2;
}

// t is tile (i0, j0) of A = X X^T (POLY = 0; also kept as plain floats) or of A A (1; becomes P = a I + b A + c A A): stored on
// both sides of the diagonal
template <int T, int POLY> __device__ inline void put_square(float (*t)[T + 1], const OrthMat &q, const OrthScalars &s, int i0, int j0)
{
    _Float16 *out = POLY ? q.P : q.A;
    for (int u = threadIdx.x; u < T * T; u += kThreads) {
        const int r = u / T, c = u % T;
        float *p = q.A32 + (size_t)(i0 + r) * q.mp + j0 + c;
        if constexpr (POLY == 1) {
            float v = s.b * *p + s.c * t[r][c];
            if (i0 + r == j0 + c && i0 + r < q.m) v += s.a;
            t[r][c] = v;
        } else {
            *p = t[r][c];
        }
    }
    __syncthreads();
    for (int u = threadIdx.x; u < T * T / 8; u += kThreads) {
        const int r = u % T, c = u / T * 8;
        float v[8], w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = t[r][c + i];
            w[i] = t[c + i][r];
        }
        put_pieces(out, i0 + r, j0 + c, q.mp / 16, v);
        if (i0 != j0) put_pieces(out, j0 + r, i0 + c, q.mp / 16, w);
    }
}

template <int T> __device__ inline void gram_tile(const OrthMat &q, const OrthScalars &s, int b, OrthLds &lds)
{
    const int split = b % q.splits, pair = b / q.splits;
    int ti, tj;
    pair_of(pair, ti, tj);
    Tile<T / 64, T / 64> t;
    const int kblocks = q.np / 16, kb0 = split * q.kbs, kb1 = min(kblocks, kb0 + q.kbs);
    t.product(q.X, ti * T, q.X, tj * T, kblocks, kb0, kb1, lds.stage);
    if (q.splits > 1) {
        t.put_part(q.part + (size_t)b * T * T);
        return;
    }
    t.spread(tile_of<T>(lds));
    put_square<T, 0>(tile_of<T>(lds), q, s, ti * T, tj * T);
}
__global__ __launch_bounds__(kThreads, 2) void orth_gram_kernel(OrthRef L, int total)
{
    __shared__ OrthLds lds;
    int b = xcd_block(blockIdx.x, gridDim.x);
    if (b >= total) return;
    const OrthMat &q = find_mat(L.mat, L.s.count, [](const OrthMat &m) { return m.gfirst; }, b);
    if (q.big) gram_tile<128>(q, L.s, b, lds);
    else gram_tile<64>(q, L.s, b, lds);
}

// adds up the runs of X X^T of the matrices that were split, in order
template <int T> __device__ inline void join_tile(const OrthMat &q, const OrthScalars &s, int pair, OrthLds &lds)
{
    int ti, tj;
    pair_of(pair, ti, tj);
    Tile<T / 64, T / 64> t;
    t.clear();
    for (int k = 0; k < q.splits; ++k) t.add_part(q.part + ((size_t)pair * q.splits + k) * T * T);
    t.spread(tile_of<T>(lds));
    put_square<T, 0>(tile_of<T>(lds), q, s, ti * T, tj * T);
}
__global__ __launch_bounds__(kThreads, 2) void orth_join_kernel(OrthRef L)
{
    __shared__ OrthLds lds;
    int b = blockIdx.x;
    // (a matrix that was not split has no workgroups here: its first is the next one's)
    const OrthMat &q = find_mat(L.mat, L.s.count, [](const OrthMat &m) { return m.jfirst; }, b);
    if (q.big) join_tile<128>(q, L.s, b, lds);
    else join_tile<64>(q, L.s, b, lds);
}

template <int T> __device__ inline void poly_tile(const OrthMat &q, const OrthScalars &s, int b, OrthLds &lds)
{
    int ti, tj;
    pair_of(b, ti, tj);
    Tile<T / 64, T / 64> t;
    t.product(q.A, ti * T, q.A, tj * T, q.mp / 16, 0, q.mp / 16, lds.stage);
    t.spread(tile_of<T>(lds));
    put_square<T, 1>(tile_of<T>(lds), q, s, ti * T, tj * T);
}
__global__ __launch_bounds__(kThreads, 2) void orth_poly_kernel(OrthRef L, int total)
{
    __shared__ OrthLds lds;
    int b = xcd_block(blockIdx.x, gridDim.x);
    if (b >= total) return;
    const OrthMat &q = find_mat(L.mat, L.s.count, [](const OrthMat &m) { return m.first[1]; }, b);
    if (q.big) poly_tile<128>(q, L.s, b, lds);
    else poly_tile<64>(q, L.s, b, lds);
}

// t, part (m0, n0) of the result of the last step, becomes O or the update of W
template <int T> __device__ inline void finish(const float (*t)[T + 1], const OrthMat &q, const OrthScalars &s, int m0, int n0)
{
    const bool tall = q.rows > q.cols;
    const int r0 = tall ? n0 : m0, c0 = tall ? m0 : n0;
    for (int u = threadIdx.x; u < T * T; u += kThreads) {
        const int r = u / T, c = u % T;
        if (r0 + r >= q.rows || c0 + c >= q.cols) continue;
        const size_t i = (size_t)(r0 + r) * q.cols + c0 + c;
        float v = tall ? t[c][r] : t[r][c];
        if (s.muon) v = orth_get(q.out, s.out_dtype, i) * s.keep - q.wscale * v;
        orth_put(q.out, s.out_dtype, i, v);
    }
}

// X <- P X, from the transposed X (Xt, or Xt2 when odd) to X and the other transposed one; last: to the result instead
template <int T> __device__ inline void apply_tile(const OrthMat &q, const OrthScalars &s, int b, int odd, int last, OrthLds &lds)
{
    const TileAt at = tile_at<T, T>(q, b);
    Tile<T / 64, T / 64> t;
    t.product(q.P, at.m0, odd ? q.Xt2 : q.Xt, at.n0, q.mp / 16, 0, q.mp / 16, lds.stage);
    t.spread(tile_of<T>(lds));
    if (last) finish<T>(tile_of<T>(lds), q, s, at.m0, at.n0);
    else emit_x<T, T>(tile_of<T>(lds), q, odd ? q.Xt : q.Xt2, at.m0, at.n0);
}
__global__ __launch_bounds__(kThreads, 2) void orth_apply_kernel(OrthRef L, int total, int odd, int last)
{
    __shared__ OrthLds lds;
    int b = xcd_block(blockIdx.x, gridDim.x);
    if (b >= total) return;
    const OrthMat &q = find_mat(L.mat, L.s.count, [](const OrthMat &m) { return m.first[2]; }, b);
    if (q.big) apply_tile<128>(q, L.s, b, odd, last, lds);
    else apply_tile<64>(q, L.s, b, odd, last, lds);
}

// no steps: X_0 is the result
__global__ __launch_bounds__(kThreads) void orth_none_kernel(OrthRef L)
{
    __shared__ float t[kOrthTile][kOrthTile + 1];
    int b = blockIdx.x;
    const OrthMat &q = find_mat(L.mat, L.s.count, [](const OrthMat &m) { return m.first[3]; }, b);
    const TileAt at = tile_at<kOrthTile, kOrthTile>(q, b);
    for (int u = threadIdx.x; u < 64 * 64; u += kThreads) {
        const int r = u / 64, c = u % 64, row = at.n0 + c, k = at.m0 + r;
        const _Float16 *p = q.Xt + ((size_t)(row >> 5) * (q.mp / 16) + (k >> 4)) * kBlockHalfs + ((row & 31) + 32 * ((k >> 3) & 1)) * 8 + (k & 7);
        t[r][c] = ((float)p[0] + (float)p[512]) / kOrthScale;
    }
    __syncthreads();
    finish<kOrthTile>(t, q, L.s, at.m0, at.n0);
}

// ---- host ----------------------------------------------------------------------------------------------------------
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Tiles of 128 x 128 read half as much for the same products, tiles of 64 x 64 waste less of a small matrix and are four times
// as many.  128 where they leave X with enough tiles for the chip's 256 compute units, and for matrices that they do not pad to
// more than half as many rows again.  The sum over columns of X X^T is split where there are too few tiles of A to fill the chip.
constexpr int kFillUnits = 512, kFewestBlocks = 16;
struct OrthPlan {
    int count;
    struct Mat {
        int m, n, mp, np, big, splits, kbs, tiles_a, tiles_x;
        size_t x, a, part, bytes;
    } mat[kOrthItems];
    size_t bytes;
};
OrthPlan plan_orth(const xconv_orth_item *items, int count)
{
    OrthPlan P{};
    P.count = count;
    auto can = [](int m) { return m > 64 && 2 * round_up(m, 128) <= 3 * m; };
    long long large = 0;
    for (int i = 0; i < count; ++i) {
        const int m = std::min(items[i].rows, items[i].cols), n = std::max(items[i].rows, items[i].cols);
        if (can(m)) large += (long long)ceil_div(m, 128) * ceil_div(n, 128);
    }
    long long blocks = 0;
    for (int i = 0; i < count; ++i) {
        OrthPlan::Mat &q = P.mat[i];
        q.m = std::min(items[i].rows, items[i].cols);
        q.n = std::max(items[i].rows, items[i].cols);
        q.big = can(q.m) && large >= 256;
        const int T = q.big ? 128 : 64;
        q.mp = round_up(q.m, T);
        q.np = round_up(q.n, T);
        const int tm = q.mp / T;
        q.tiles_a = tm * (tm + 1) / 2;
        q.tiles_x = tm * (q.np / T);
        blocks += (long long)q.tiles_a * (q.np / 16);
    }
    // runs of about as many blocks as give every compute unit two workgroups
    const int run = (int)std::max<long long>(kFewestBlocks, round_up((int)std::min<long long>((blocks + kFillUnits - 1) / kFillUnits, 1 << 20), 4));
    P.bytes = up256(sizeof(OrthMat) * kOrthItems);
    for (int i = 0; i < count; ++i) {
        OrthPlan::Mat &q = P.mat[i];
        const int kb = q.np / 16;
        q.splits = kb >= 2 * run ? ceil_div(kb, run) : 1;
        q.kbs = q.splits > 1 ? run : kb;
        q.x = up256((size_t)q.mp * q.np * 4);
        q.a = up256((size_t)q.mp * q.mp * 4);
        q.part = q.splits > 1 ? up256((size_t)q.tiles_a * q.splits * (q.big ? 128 * 128 : 64 * 64) * 4) : 0;
        q.bytes = 3 * q.x + 3 * q.a + q.part + up256(kOrthNorms * sizeof(double));
        P.bytes += q.bytes;
    }
    return P;
}

}  // namespace

// the matrices go through in runs of kOrthItems, one run after the other through the same scratch
size_t orth_ws_bytes(const xconv_orth_item *items, int count)
{
    size_t most = 256;
    for (int at = 0; at < count; at += kOrthItems) most = std::max(most, plan_orth(items + at, std::min(kOrthItems, count - at)).bytes);
    return most;
}

hipError_t launch_orth(const xconv_orth_item *items, int count, const xconv_orth_args *args, const xconv_muon_args *muon, void *ws, hipStream_t st)
{
    for (int at = 0; at < count; at += kOrthItems) {
        const OrthPlan P = plan_orth(items + at, std::min(kOrthItems, count - at));
        OrthList L{};
        OrthScalars &s = L.s;
        s.count = P.count;
        s.g_dtype = args->g_dtype; s.out_dtype = args->out_dtype;
        s.a = args->a; s.b = args->b; s.c = args->c; s.eps = args->eps;
        if (muon) {
            s.muon = 1; s.nesterov = muon->nesterov != 0; s.mu = muon->momentum;
            s.keep = (float)(1.0 - (double)muon->lr * muon->weight_decay);
        }
        char *p = static_cast<char *>(ws);
        auto take = [&](size_t bytes) { char *r = p; p += bytes; return r; };
        OrthMat *list = (OrthMat *)take(up256(sizeof(OrthMat) * kOrthItems));
        int total[4] = {0, 0, 0, 0}, gram = 0, join = 0;
        for (int i = 0; i < P.count; ++i) {
            const xconv_orth_item &it = items[at + i];
            const OrthPlan::Mat &f = P.mat[i];
            OrthMat &q = L.mat[i];
            q.G = it.G_dev; q.out = it.out_dev; q.M = it.M_dev;
            q.rows = it.rows; q.cols = it.cols; q.m = f.m; q.n = f.n; q.mp = f.mp; q.np = f.np;
            q.big = f.big; q.splits = f.splits; q.kbs = f.kbs;
            q.X = (_Float16 *)take(f.x); q.Xt = (_Float16 *)take(f.x); q.Xt2 = (_Float16 *)take(f.x);
            q.A = (_Float16 *)take(f.a); q.P = (_Float16 *)take(f.a); q.A32 = (float *)take(f.a);
            q.part = (float *)take(f.part);
            q.sq = (double *)take(up256(kOrthNorms * sizeof(double)));
            q.nsq = (int)std::min<size_t>(kOrthNorms, ((size_t)it.rows * it.cols + 4095) / 4096);
            if (muon) q.wscale = (float)((double)muon->lr * std::sqrt(std::max(1.0, (double)it.rows / it.cols)));
            const int blocks[4] = {q.nsq, f.tiles_a, f.tiles_x, (f.mp / kOrthTile) * (f.np / kOrthTile)};
            for (int k = 0; k < 4; ++k) {
                q.first[k] = total[k];
                total[k] += blocks[k];
            }
            q.gfirst = gram;
            gram += f.tiles_a * f.splits;
            q.jfirst = join;
            join += f.splits > 1 ? f.tiles_a : 0;
        }
        const OrthRef R{s, list};
        const dim3 block(kThreads);
        auto grid8 = [](int n) { return dim3((unsigned)round_up(n, 8)); };
        hipLaunchKernelGGL(orth_norm_kernel, dim3(total[0]), block, 0, st, L, list);
        hipLaunchKernelGGL(orth_start_kernel, dim3(total[3]), block, 0, st, R);
        if (args->steps == 0) hipLaunchKernelGGL(orth_none_kernel, dim3(total[3]), block, 0, st, R);
        for (int k = 0; k < args->steps; ++k) {
            hipLaunchKernelGGL(orth_gram_kernel, grid8(gram), block, 0, st, R, gram);
            if (join) hipLaunchKernelGGL(orth_join_kernel, dim3(join), block, 0, st, R);
            hipLaunchKernelGGL(orth_poly_kernel, grid8(total[1]), block, 0, st, R, total[1]);
            hipLaunchKernelGGL(orth_apply_kernel, grid8(total[2]), block, 0, st, R, total[2], k & 1, k + 1 == args->steps);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace xc
