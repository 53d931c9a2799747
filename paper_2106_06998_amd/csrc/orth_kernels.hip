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
//
// Three ways, by the matrix' own extents: up to 64 x 768 all steps in one workgroup (orth_narrow_kernel); up to 256 rows two launches
// a step, X X^T and both products by A (orth_merge_kernel); else three, X X^T, P and P X, in tiles of 64 x 64 or 128 x 128.  Wide
// matrices of 128 rows and 2^18 values or more take only the first and the last of these three once for up to three steps (see `grouped`).  The sums
// of X X^T and A A are split along k where their tiles are too few for the chip and joined in order by another launch.  What else
// is in a call changes the tiles but not one bit of a result.
//
// Measured, five steps: 64 x 576 fp32 44 us (7.2 us a step, most of it one compute unit's matrix instructions), 200 x 147 88 us
// (two launches of 6 to 9 us a step), 2048 x 4096 fp32 1.02 ms (three fp16 products for one: 0.8 to 0.98 PFLOP/s of them in the
// large products, where a large library product reaches 1.2), 8 of 512 x 4608 bf16 with the weights' update 0.60 ms.
#include <algorithm>
#include <cmath>
#include <mutex>
#include <new>

#include "common.h"
#include "launch.h"

namespace xc {

namespace {

constexpr float kOrthScale = 4096.f, kOrthUnscale = 1.f / (4096.f * 4096.f);
constexpr int kOrthItems = 24;      // matrices of one launch (as many as kernel arguments hold)
constexpr int kOrthTile = 64;       // extents are padded to this or twice this
constexpr int kOrthNorms = 512;     // most partial sums of a matrix' squares
constexpr int kBlockHalfs = 1024;   // 32 x 16 values, both numbers

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct OrthMat {
    const void *G;
    void *out;
    float *M;
    _Float16 *X, *Xt, *Xt2, *S;         // fragment order; S: A and the other symmetric matrices, one after the other
    double *sq;                         // partial sums of squares
    float *part;                        // partial products of X X^T, [tile][split][tile values]
    int rows, cols, m, n, mp, np;       // m <= n
    int nsq;
    int big[3];                         // tiles of 128 x 128 (else 64 x 64) of A, of P, of X
    int gsplits, gkbs, psplits, pkbs;   // X X^T and A A: runs of blocks of 16 along the sum, and their length
    float wscale;                       // lr sqrt(max(1, rows / cols))
};
struct OrthScalars {
    int count, g_dtype, out_dtype, muon, nesterov;
    float a, b, c, eps, mu, rest, keep;     // rest = 1 - mu, keep = 1 - lr decay, both rounded once from 64 bits
};
struct OrthList {
    OrthScalars s;
    int first[kOrthItems];
    OrthMat mat[kOrthItems];
};
static_assert(sizeof(OrthList) <= 4096, "kernel arguments");
// A product of two symmetric matrices S_left S_right, symmetric itself, goes to S_out times `scale`
struct Squares {
    int left, right, out;
    float scale;
};
// What the launches after the first are given: the list lies in the scratch
struct OrthRef {
    OrthScalars s;
    int total;                          // workgroups that have work
    int first[kOrthItems];              // each matrix' first workgroup
    const OrthMat *mat;
    OrthMat one;                        // the matrix of a list of one
};

// which matrix workgroup b belongs to (one without workgroups starts where the next one does); b becomes its number in there
__device__ inline int find_mat(const int *first, int count, int &b)
{
    int lo = 0, hi = count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= b) lo = mid;
        else hi = mid - 1;
    }
    b -= first[lo];
    return lo;
}

__device__ inline OrthMat the_mat(const OrthRef &L, int &b)
{
    if (L.s.count == 1) return L.one;
    return L.mat[find_mat(L.first, L.s.count, b)];
}

__device__ inline _Float16 *square_of(const OrthMat &q, int k) { return q.S + (size_t)k * q.mp * q.mp * 2; }

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
// N values whose places `at(k)` gives, zero where it is negative: one branch on the type for all of them, so that the loads go
// out together
__device__ inline float half_value(uint16_t h, bool bf) { return bf ? bf16_to_f32(h) : f16_to_f32(h); }
template <int N, class At> __device__ inline void orth_gather(const void *p, int dtype, At &&at, float (&v)[N])
{
    if (dtype == XCONV_F32) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const auto i = at(k);
            v[k] = static_cast<const float *>(p)[i < 0 ? 0 : i];
        }
    } else {
        uint16_t h[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const auto i = at(k);
            h[k] = static_cast<const uint16_t *>(p)[i < 0 ? 0 : i];
        }
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = half_value(h[k], dtype == XCONV_BF16);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = at(k) < 0 ? 0.f : v[k];
}
// the same of a matrix and of one of floats, all loads together
template <int N, class At> __device__ inline void orth_gather2(const void *p, int dtype, const float *p2, At &&at, float (&v)[N], float (&v2)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const auto i = at(k);
        v2[k] = p2[i < 0 ? 0 : i];
    }
    orth_gather(p, dtype, at, v);
#pragma unroll
    for (int k = 0; k < N; ++k) v2[k] = at(k) < 0 ? 0.f : v2[k];
}
__device__ inline float update_of(float g, float m, const OrthScalars &L) { return L.nesterov ? g + L.mu * (m - g) : m; }

// eight values, already scaled, as two fp16 numbers each (rounded to nearest; the rest of the first is exact)
__device__ inline void split8(const float (&s)[8], h8 &h, h8 &l)
{
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const h2 hi = __builtin_convertvector(f32x2{s[i], s[i + 1]}, h2);
        f32x2 rest;
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(rest[0]) : "v"(hi), "v"(s[i]));
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(rest[1]) : "v"(hi), "v"(s[i + 1]));
        const h2 lo = __builtin_convertvector(rest, h2);
        h[i] = hi[0]; h[i + 1] = hi[1];
        l[i] = lo[0]; l[i + 1] = lo[1];
    }
}
// where row r, columns k .. k + 7 of a matrix in fragment order lie (the second numbers 512 values on)
template <class H> __device__ inline H *place_of(H *frag, int r, int k, int kblocks)
{
    return frag + ((size_t)(r >> 5) * kblocks + (k >> 4)) * kBlockHalfs + ((r & 31) + 32 * ((k >> 3) & 1)) * 8;
}
__device__ inline void put_pieces(_Float16 *frag, int r, int k, int kblocks, const float (&v)[8])
{
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = v[i] * kOrthScale;
    h8 h, l;
    split8(s, h, l);
    _Float16 *p = place_of(frag, r, k, kblocks);
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

// eight values from element i on, as they are (16 bits: in the first vector) and as floats
struct __attribute__((packed, aligned(2))) Loose8 { uint32_t w[4]; };
__device__ inline void raw_get8(const void *p, int dtype, size_t i, u32x4 (&v)[2])
{
    if (dtype == XCONV_F32) {
        const Loose4 *q = reinterpret_cast<const Loose4 *>(static_cast<const float *>(p) + i);
        const Loose4 a = q[0], b = q[1];
        v[0] = u32x4{a.w[0], a.w[1], a.w[2], a.w[3]};
        v[1] = u32x4{b.w[0], b.w[1], b.w[2], b.w[3]};
    } else {
        const Loose8 a = *reinterpret_cast<const Loose8 *>(static_cast<const uint16_t *>(p) + i);
        v[0] = u32x4{a.w[0], a.w[1], a.w[2], a.w[3]};
    }
}
__device__ inline void raw_values(const u32x4 (&r)[2], int dtype, float (&v)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k)
        v[k] = dtype == XCONV_F32 ? __uint_as_float(r[k >> 2][k & 3]) : half_value((uint16_t)(r[0][k >> 1] >> (16 * (k & 1))), dtype == XCONV_BF16);
}
__device__ inline void orth_put8(void *p, int dtype, size_t i, const float (&v)[8])
{
    if (dtype == XCONV_F32) {
        Loose4 *q = reinterpret_cast<Loose4 *>(static_cast<float *>(p) + i);
        q[0] = Loose4{{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}};
        q[1] = Loose4{{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])}};
        return;
    }
    Loose8 h;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        h.w[k] = dtype == XCONV_BF16 ? bf16_pair(v[2 * k], v[2 * k + 1]) : __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2 * k], v[2 * k + 1]}, h2));
    *reinterpret_cast<Loose8 *>(static_cast<uint16_t *>(p) + i) = h;
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
    const OrthMat &q = L.mat[find_mat(L.first, L.s.count, b)];
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
                m[k] = m[k] + (u[k] - m[k]) * L.s.rest;
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
// the same for all rows and TN columns from n0 on, where the matrix may have fewer than TM rows
template <int TM, int TN, int NTHR> __device__ inline void emit_rows(const float (*t)[TN + 1], const OrthMat &q, _Float16 *xt, int n0)
{
    for (int u = threadIdx.x; u < TM * TN / 8; u += NTHR) {
        float v[8];
        int r = u % TM, c = u / TM * 8;
        if (r < q.mp) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = t[r][c + i];
            put_pieces(q.X, r, n0 + c, q.np / 16, v);
        }
        r = u / TN * 8;
        c = u % TN;
        if (r < q.mp) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = t[r + i][c];
            put_pieces(xt, n0 + c, r, q.mp / 16, v);
        }
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
    const OrthMat q = the_mat(L, b);
    const TileAt at = tile_at<kOrthTile, kOrthTile>(q, b);
    const bool tall = q.rows > q.cols;
    const int r0 = tall ? at.n0 : at.m0, c0 = tall ? at.m0 : at.n0;
    constexpr int kRound = 16;
    float v[kRound], m[kRound];
    auto place = [&](int k) -> long long {
        const int u = k * kThreads + threadIdx.x, r = r0 + u / kOrthTile, c = c0 + u % kOrthTile;
        return r < q.rows && c < q.cols ? (long long)r * q.cols + c : -1;
    };
    if (L.s.muon) {
        orth_gather2(q.G, L.s.g_dtype, q.M, place, v, m);
#pragma unroll
        for (int k = 0; k < kRound; ++k) v[k] = update_of(v[k], m[k], L.s);
    } else {
        orth_gather(q.G, L.s.g_dtype, place, v);
    }
    const double norm = sqrt(sum_squares(q)), d = norm < (double)L.s.eps ? (double)L.s.eps : norm;      // (a NaN stays one)
    const double inv = d == 0.0 ? 0.0 : 1.0 / d;                                                         // (eps = 0 and a zero matrix)
#pragma unroll
    for (int k = 0; k < kRound; ++k) {
        const int u = k * kThreads + threadIdx.x, r = u / kOrthTile, c = u % kOrthTile;
        const float x = place(k) >= 0 ? (float)((double)v[k] * inv) : 0.f;
        if (tall) t[c][r] = x;
        else t[r][c] = x;
    }
    __syncthreads();
    emit_x<kOrthTile, kOrthTile>(t, q, q.Xt, at.m0, at.n0);
}

// ---- products ------------------------------------------------------------------------------------------------------
// A workgroup's tile: 64 MT rows of one matrix times 64 NT rows of another (rows along k, fragment order with kblocks blocks a
// row of blocks), blocks kb0 .. kb1 - 1; wave w computes rows 32 MT (w / 2), columns 32 NT (w % 2).  Steps of KS blocks.  The first
// matrix' fragments go through LDS (staged through registers into one of two buffers while the other one is used: one barrier a
// step), the second one's straight into the registers of the two waves that use them, a step ahead: both ways through LDS, its
// bandwidth is what the matrix instructions wait for.
template <int MT, int NT> struct Tile {
    static constexpr int TM = 64 * MT, TN = 64 * NT, KS = 2, kUnits = 2 * MT * KS * 128, kPer = kUnits / kThreads;
    f32x16 acc[MT][NT];
    struct Right {
        h8 f[KS][2][NT];
    };

    __device__ void clear()
    {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    }
    __device__ static void load(u32x4 (&r)[kPer], const _Float16 *Fa, int ra, int kblocks, int kb)
    {
        constexpr int kRun = KS * 128;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            // (a run is a whole number of rounds of the workgroup)
            const int blk = j * kThreads / kRun, off = (j * kThreads) % kRun + (int)threadIdx.x;
            r[j] = reinterpret_cast<const u32x4 *>(Fa + ((size_t)(ra / 32 + blk) * kblocks + kb) * kBlockHalfs)[off];
        }
    }
    __device__ static void load(Right &r, const _Float16 *Fb, int rb, int kblocks, int kb)
    {
        const int wb = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) & 1), lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int p = 0; p < 2; ++p)
                    r.f[k][p][j] = reinterpret_cast<const h8 *>(Fb + ((size_t)(rb / 32 + wb * NT + j) * kblocks + kb + k) * kBlockHalfs + p * 512)[lane];
    }
    __device__ static void store(const u32x4 (&r)[kPer], u32x4 *lds)
    {
#pragma unroll
        for (int j = 0; j < kPer; ++j) lds[j * kThreads + threadIdx.x] = r[j];
    }
    __device__ void multiply(const u32x4 *lds, const Right &b)
    {
        const int wa = threadIdx.x >> 7, lane = threadIdx.x & 63;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            h8 a[2][MT];
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < MT; ++i) a[p][i] = __builtin_bit_cast(h8, lds[((wa * MT + i) * KS + k) * 128 + p * 64 + lane]);
            // the small products first
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[p == 0][i], b.f[k][p == 1][j], acc[i][j], 0, 0, 0);
        }
    }
    // 64 x 64: every wave loads its own fragments, four blocks ahead of the ones that it multiplies
    __device__ void product_direct(const _Float16 *Fa, int ra, const _Float16 *Fb, int rb, int kblocks, int kb0, int kb1)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
        const h8 *pa = reinterpret_cast<const h8 *>(Fa + ((size_t)(ra / 32 + (wave >> 1)) * kblocks + kb0) * kBlockHalfs) + lane;
        const h8 *pb = reinterpret_cast<const h8 *>(Fb + ((size_t)(rb / 32 + (wave & 1)) * kblocks + kb0) * kBlockHalfs) + lane;
        h8 a[2][4][2], b[2][4][2];
        auto get = [&](int s) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    a[s][k][p] = pa[k * 128 + p * 64];
                    b[s][k][p] = pb[k * 128 + p * 64];
                }
            pa += 4 * 128;
            pb += 4 * 128;
        };
        auto use = [&](int s) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[s][k][1], b[s][k][0], acc[0][0], 0, 0, 0);
                acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[s][k][0], b[s][k][1], acc[0][0], 0, 0, 0);
                acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[s][k][0], b[s][k][0], acc[0][0], 0, 0, 0);
            }
        };
        clear();
        int left = (kb1 - kb0) / 4;
        get(0);
        if (left > 1) get(1);
#pragma unroll 1
        for (; left > 2; left -= 2) {
            use(0);
            get(0);
            use(1);
            if (left > 3) get(1);
        }
        use(0);
        if (left > 1) use(1);
    }
    // lds: two steps
    __device__ void product(const _Float16 *Fa, int ra, const _Float16 *Fb, int rb, int kblocks, int kb0, int kb1, u32x4 *lds)
    {
        clear();
        u32x4 r[kPer];
        Right b0, b1;
        load(b0, Fb, rb, kblocks, kb0);
        load(r, Fa, ra, kblocks, kb0);
        store(r, lds);
        __syncthreads();
        int at = 0;
        // one step with the next one's loads under way
        auto step = [&](const Right &now, Right &next, int kb) {
            load(next, Fb, rb, kblocks, kb);
            load(r, Fa, ra, kblocks, kb);
            multiply(lds + at * kUnits, now);
            at ^= 1;
            store(r, lds + at * kUnits);
            __syncthreads();
        };
        int kb = kb0 + KS;
        for (; kb + KS < kb1; kb += 2 * KS) {
            step(b0, b1, kb);
            step(b1, b0, kb + KS);
        }
        if (kb < kb1) {
            step(b0, b1, kb);
            multiply(lds + at * kUnits, b1);
        } else {
            multiply(lds + at * kUnits, b0);
        }
        __syncthreads();
    }
    // the sums, in true scale (times a factor), as t[row][column]
    __device__ void spread(float (*t)[TN + 1], float factor = 1.f) const
    {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        const float unscale = kOrthUnscale * factor;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    t[32 * (MT * (wave >> 1) + i) + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)][32 * (NT * (wave & 1) + j) + (lane & 31)] = acc[i][j][e] * unscale;
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

// A workgroup's LDS: two steps of the product, then the tile of the result
template <int T> union TileLds {
    u32x4 stage[T == 64 ? 1 : 2 * Tile<T / 64, T / 64>::kUnits];
    float t[T][T + 1];
};
// A tile's product: of 64 x 64 straight from memory, which a small matrix' few workgroups get through sooner; of 128 x 128 through
// LDS, which takes less from the caches
template <int T> __device__ inline void tile_of_product(TileLds<T> &lds, Tile<T / 64, T / 64> &t, const _Float16 *Fa, int ra, const _Float16 *Fb, int rb,
                                                        int kblocks, int kb0, int kb1)
{
    if constexpr (T == 64) t.product_direct(Fa, ra, Fb, rb, kblocks, kb0, kb1);
    else t.product(Fa, ra, Fb, rb, kblocks, kb0, kb1, lds.stage);
}

// pair (i <= j) of tiles of a symmetric matrix with T rows of tiles
__device__ inline void pair_of(int b, int &i, int &j)
{
    j = (int)((sqrtf(8.f * (float)b + 1.f) - 1.f) * 0.5f);
    while ((j + 1) * (j + 2) / 2 <= b) ++j;
    while (j * (j + 1) / 2 > b) --j;
    i = b - j * (j + 1) / 2;
}

// What a product of symmetric tiles is: A = X X^T, P = a I + b A + c A A, or a product of two polynomials of X X^T
enum { GRAM, POLY, MUL };

// t is part of A (GRAM), of A A (POLY: P is stored) or of a product (MUL).  Its rows are i0 on
// and its columns j0 on (STEP = 32), or, when it is the part (i, j) of a tile of 128, every other run of 32 of them (STEP = 64).
// What lies on and above the diagonal blocks of 32 x 32 is stored on both sides of the diagonal, so that A and P are symmetric
// to the last bit whatever the tiles.
template <int T, int KIND, int STEP> __device__ inline void put_square(float (*t)[T + 1], const OrthMat &q, const OrthScalars &s, const Squares &u, int i0, int j0)
{
    _Float16 *out = square_of(q, u.out);
    const _Float16 *A = square_of(q, u.left);
    auto along = [](int from, int r) { return from + STEP * (r >> 5) + (r & 31); };
    // eight values of the result, A A's being v, at (row, col) and right of it
    auto put = [&](int row, int col, float (&v)[8]) {
        if constexpr (KIND == POLY) {
            const _Float16 *p = place_of(A, row, col, q.mp / 16);
            const h8 h = *reinterpret_cast<const h8 *>(p), l = *reinterpret_cast<const h8 *>(p + 512);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = s.b * (((float)h[i] + (float)l[i]) * (1.f / kOrthScale)) + s.c * v[i];
                if (row == col + i && row < q.m) v[i] += s.a;
            }
        }
        put_pieces(out, row, col, q.mp / 16, v);
    };
    for (int i = threadIdx.x; i < T * T / 8; i += kThreads) {
        const int r = i % T, c = i / T * 8;
        float v[8];
        {
            const int row = along(i0, r), col = along(j0, c);
            const bool diagonal = row >> 5 == col >> 5;
            if (row >> 5 <= col >> 5) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = diagonal && (c + i & 31) < (r & 31) ? t[(r & ~31) + (c + i & 31)][(c & ~31) + (r & 31)] : t[r][c + i];
                put(row, col, v);
            }
        }
        {
            // (r runs along the columns here)
            const int row = along(i0, c), col = along(j0, r);
            if (row >> 5 < col >> 5) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = t[c + i][r];
                put(col, row, v);
            }
        }
    }
}

// a workgroup: a pair of rows of tiles and a run along the sum
template <int T, int KIND> __global__ __launch_bounds__(kThreads, 2) void orth_square_kernel(OrthRef L, Squares u)
{
    __shared__ TileLds<T> lds;
    int b = xcd_block(blockIdx.x, gridDim.x);
    if (b >= L.total) return;
    const OrthMat q = the_mat(L, b);
    const bool gram = KIND == GRAM;
    const int splits = gram ? q.gsplits : q.psplits, run = gram ? q.gkbs : q.pkbs, kblocks = (gram ? q.np : q.mp) / 16;
    const int split = b % splits, pair = b / splits;
    const _Float16 *left = gram ? q.X : square_of(q, u.left), *right = gram ? q.X : square_of(q, u.right);
    int ti, tj;
    pair_of(pair, ti, tj);
    Tile<T / 64, T / 64> t;
    tile_of_product<T>(lds, t, left, ti * T, right, tj * T, kblocks, split * run, min(kblocks, (split + 1) * run));
    if (splits > 1) {
        t.put_part(q.part + (size_t)b * T * T);
        return;
    }
    t.spread(lds.t, u.scale);
    put_square<T, KIND, 32>(lds.t, q, L.s, u, ti * T, tj * T);
}

// adds up the runs of a product, in order: 64 x 64 values a workgroup
template <int KIND> __global__ __launch_bounds__(kThreads) void orth_join_kernel(OrthRef L, Squares u)
{
    __shared__ float t[64][64 + 1];
    int b = blockIdx.x;
    const OrthMat q = the_mat(L, b);
    const bool big = q.big[KIND == GRAM ? 0 : 1];
    const int splits = KIND == GRAM ? q.gsplits : q.psplits, parts = big ? 4 : 1, pair = b / parts, part = b % parts;
    int ti, tj;
    pair_of(pair, ti, tj);
    Tile<1, 1> sum;
    sum.clear();
    for (int k = 0; k < splits; ++k) sum.add_part(q.part + ((size_t)(pair * splits + k) * parts + part) * 64 * 64);
    sum.spread(t, u.scale);
    if (big) put_square<64, KIND, 64>(t, q, L.s, u, ti * 128 + 32 * (part >> 1), tj * 128 + 32 * (part & 1));
    else put_square<64, KIND, 32>(t, q, L.s, u, ti * 64, tj * 64);
}

// Part (m0, n0) of the result of the last step becomes O or the update of W: eight values in the order of memory a thread and
// round, four threads a row.  The weights are loaded for all rounds before the first is needed.
template <int TM, int TN, int NTHR = kThreads> struct Finish {
    static constexpr int N = TM * TN / 8 / NTHR;
    const OrthMat &q;
    const OrthScalars &s;
    bool tall;
    int r0, c0;
    u32x4 w[N][2];

    __device__ Finish(const OrthMat &q, const OrthScalars &s, int m0, int n0) : q(q), s(s)
    {
        tall = q.rows > q.cols;
        r0 = tall ? n0 : m0;
        c0 = tall ? m0 : n0;
    }
    __device__ int row(int j) const
    {
        const int u = (j * NTHR + (int)threadIdx.x) / 4;
        return tall ? u % TN : u % TM;
    }
    __device__ int col(int j) const
    {
        const int u = (j * NTHR + (int)threadIdx.x) / 4;
        return ((tall ? u / TN : u / TM) * 4 + (int)threadIdx.x % 4) * 8;
    }
    // how many of the eight there are, and the first one's place
    __device__ int there(int j) const { return r0 + row(j) < q.rows ? max(0, min(8, q.cols - (c0 + col(j)))) : 0; }
    __device__ size_t place(int j) const { return (size_t)(r0 + row(j)) * q.cols + c0 + col(j); }
    __device__ void load()
    {
        if (!s.muon) return;
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (there(j) == 8) raw_get8(q.out, s.out_dtype, place(j), w[j]);
    }
    __device__ void put(const float (*t)[TN + 1])
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int n = there(j), r = row(j), c = col(j);
            if (n == 8) {
                float v[8], old[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = tall ? t[c + k][r] : t[r][c + k];
                if (s.muon) {
                    raw_values(w[j], s.out_dtype, old);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = old[k] * s.keep - q.wscale * v[k];
                }
                orth_put8(q.out, s.out_dtype, place(j), v);
            } else {
#pragma unroll 1
                for (int k = 0; k < n; ++k) {
                    float v = tall ? t[c + k][r] : t[r][c + k];
                    if (s.muon) v = orth_get(q.out, s.out_dtype, place(j) + k) * s.keep - q.wscale * v;
                    orth_put(q.out, s.out_dtype, place(j) + k, v);
                }
            }
        }
    }
};

// X <- P X, P being `scale` times S_which, from the transposed X (Xt, or Xt2 when odd) to X and the other transposed one.  LAST: to the result instead.
// All three products for results of 16 bits too: the first numbers' product alone takes 8 of 512 x 4608 from 603 to 580 us, but it is
// 3e-4 of O away, more than rounding to fp16, and for a falling spectrum as far as rounding to bf16.
template <int T, int LAST> __global__ __launch_bounds__(kThreads, 2) void orth_apply_kernel(OrthRef L, int odd, int which, float scale)
{
    __shared__ TileLds<T> lds;
    int b = xcd_block(blockIdx.x, gridDim.x);
    if (b >= L.total) return;
    const OrthMat q = the_mat(L, b);
    const TileAt at = tile_at<T, T>(q, b);
    Tile<T / 64, T / 64> t;
    tile_of_product<T>(lds, t, square_of(q, which), at.m0, odd ? q.Xt2 : q.Xt, at.n0, q.mp / 16, 0, q.mp / 16);
    if constexpr (LAST) {
        Finish<T, T> f(q, L.s, at.m0, at.n0);
        f.load();
        t.spread(lds.t, scale);
        f.put(lds.t);
    } else {
        t.spread(lds.t, scale);
        emit_x<T, T>(lds.t, q, odd ? q.Xt : q.Xt2, at.m0, at.n0);
    }
}

// ---- matrices of up to 256 rows: X <- a X + A (b X + c A X) in one launch -------------------------------------------
// P costs such a matrix a launch of a few workgroups, which is latency (200 x 147: 7 us for P and 5 us for P X; this launch takes 9).
// Here a workgroup takes 32 CB columns of X through both
// products by A: wave w holds rows 32 w .. of A in registers (read once, all loads together), the columns of X and then
// Z = b X + c A X lie in LDS as the second operand, and a X is where the second product's sums start from.
template <int MB, int CB> union MergeLds {
    u32x4 frag[CB][2 * MB * 128];
    float t[32 * MB][32 * CB + 1];
};
template <int MB, int CB, int LAST> __global__ __launch_bounds__(64 * MB, MB == 8 ? 2 : 1) void orth_merge_kernel(OrthRef L, int odd)
{
    extern __shared__ char merge_lds[];
    MergeLds<MB, CB> &lds = *reinterpret_cast<MergeLds<MB, CB> *>(merge_lds);
    constexpr int KB = 2 * MB, NTHR = 64 * MB;
    int b = blockIdx.x;
    const OrthMat q = the_mat(L, b);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int n0 = b * 32 * CB, kblocks = q.mp / 16;
    const bool mine = 32 * wave < q.mp;          // (waves past the matrix' rows only help to copy)
    // columns n0 .. of X, which are rows of the transposed X: whole kilobytes
    const u32x4 *x = reinterpret_cast<const u32x4 *>((odd ? q.Xt2 : q.Xt) + (size_t)(n0 / 32) * kblocks * kBlockHalfs);
    u32x4 r[CB * KB * 128 / NTHR];
    const int units = kblocks * 128;
#pragma unroll
    for (int j = 0; j < CB * KB * 128 / NTHR; ++j) r[j] = j * NTHR + tid < CB * units ? x[j * NTHR + tid] : u32x4{0, 0, 0, 0};
    h8 a[KB][2];
    if (mine) {
        const h8 *f = reinterpret_cast<const h8 *>(q.S + (size_t)wave * kblocks * kBlockHalfs) + lane;
#pragma unroll
        for (int k = 0; k < KB; ++k)
            if (k < kblocks) {
                a[k][0] = f[k * 128];
                a[k][1] = f[k * 128 + 64];
            }
    }
    u32x4 *frag = &lds.frag[0][0];               // [column block][block along k][number][lane], of the matrix' own extent
#pragma unroll
    for (int j = 0; j < CB * KB * 128 / NTHR; ++j)
        if (j * NTHR + tid < CB * units) frag[j * NTHR + tid] = r[j];
    __syncthreads();
    f32x16 acc[CB];
    auto product = [&] {
#pragma unroll
        for (int k = 0; k < KB; ++k)
            if (k < kblocks) {
                h8 v[CB][2];
#pragma unroll
                for (int j = 0; j < CB; ++j)
#pragma unroll
                    for (int p = 0; p < 2; ++p) v[j][p] = __builtin_bit_cast(h8, frag[j * units + k * 128 + p * 64 + lane]);
#pragma unroll
                for (int p = 0; p < 3; ++p)
#pragma unroll
                    for (int j = 0; j < CB; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[k][p == 0], v[j][p == 1], acc[j], 0, 0, 0);
            }
    };
#pragma unroll
    for (int j = 0; j < CB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[j][e] = 0.f;
    // registers 4 g .. of a lane are four of the eight values of one lane's fragment: its place in LDS
    auto four = [&](int j, int g, int p) {
        const int k = 2 * wave + (g >> 1), from = (lane & 31) + 32 * (g & 1);
        return reinterpret_cast<h4 *>(frag + j * units + k * 128 + p * 64 + from) + (lane >> 5);
    };
    h4 zh[CB][4], zl[CB][4];
    if (mine) {
        product();
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const h4 xh = *four(j, g, 0), xl = *four(j, g, 1);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // (X scaled once, the sums twice)
                    const float v = (float)xh[i] + (float)xl[i], z = L.s.b * v + L.s.c * (acc[j][4 * g + i] * (1.f / kOrthScale));
                    zh[j][g][i] = (_Float16)z;
                    zl[j][g][i] = (_Float16)(z - (float)zh[j][g][i]);
                    acc[j][4 * g + i] = L.s.a * v * kOrthScale;
                }
            }
    }
    __syncthreads();
    if (mine) {
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                *four(j, g, 0) = zh[j][g];
                *four(j, g, 1) = zl[j][g];
            }
    }
    __syncthreads();
    if (mine) product();
    __syncthreads();
    if (mine) {
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) lds.t[32 * wave + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)][32 * j + (lane & 31)] = acc[j][e] * kOrthUnscale;
    }
    if constexpr (LAST) {
        Finish<32 * MB, 32 * CB, NTHR> f(q, L.s, 0, n0);
        f.load();
        __syncthreads();
        f.put(lds.t);
    } else {
        __syncthreads();
        emit_rows<32 * MB, 32 * CB, NTHR>(lds.t, q, odd ? q.Xt : q.Xt2, n0);
    }
}

// no steps: X_0 is the result
__global__ __launch_bounds__(kThreads) void orth_none_kernel(OrthRef L)
{
    __shared__ float t[kOrthTile][kOrthTile + 1];
    int b = blockIdx.x;
    const OrthMat q = the_mat(L, b);
    const TileAt at = tile_at<kOrthTile, kOrthTile>(q, b);
    for (int u = threadIdx.x; u < 64 * 64; u += kThreads) {
        const int r = u / 64, c = u % 64, row = at.n0 + c, k = at.m0 + r;
        const _Float16 *p = q.Xt + ((size_t)(row >> 5) * (q.mp / 16) + (k >> 4)) * kBlockHalfs + ((row & 31) + 32 * ((k >> 3) & 1)) * 8 + (k & 7);
        t[r][c] = ((float)p[0] + (float)p[512]) / kOrthScale;
    }
    __syncthreads();
    Finish<kOrthTile, kOrthTile> f(q, L.s, at.m0, at.n0);
    f.load();
    f.put(t);
}

// ---- small matrices: all steps in one workgroup -------------------------------------------------------------------
// m <= 64 and n <= 768: eight waves hold X in registers, 64 rows x 32 columns a tile and up to three tiles a wave, in the layout
// in which the matrix instruction leaves its result: a lane has one column of 32 and half of the rows.  Read as an operand, that
// is the column's part of P X (k runs over rows, in the order in which the lane has them; P is laid out in the same order), and
// with the operands changed over it gives the same product transposed, a lane having one row of A and columns along k, which
// is what X X^T takes.  So X never leaves the registers; the waves' parts of X X^T are added up through LDS.
// What bounds it is latency and one unit's matrix instructions (64 x 576: 44 us; with a launch a product, 15 of them, 115 us).
constexpr int kNarrowThreads = 512, kNarrowWaves = 8, kNarrowTiles = 3, kNarrowItems = 64;
constexpr int kNarrowM = 64, kNarrowN = 32 * kNarrowWaves * kNarrowTiles;

struct NarrowMat {
    const void *G;
    void *out;
    float *M;
    int rows, cols;
    float wscale;
};
struct NarrowList {
    OrthScalars s;
    int steps;
    NarrowMat mat[kNarrowItems];
};
static_assert(sizeof(NarrowList) <= 4096, "kernel arguments");

struct NarrowLds {
    union {
        f32x4 gram[kNarrowWaves][4][4][64];     // [wave][block][registers / 4][lane] of X X^T
        double red[kNarrowWaves];
    };
    h8 af[2][2][2][2][64], pf[2][2][2][2][64];  // A and P: [rows / 32][k / 32][half][number][lane]
};
static_assert(sizeof(NarrowLds) <= 160 * 1024, "LDS of a compute unit");

// registers 8 kq .. 8 kq + 7 of a result, scaled, as an operand
__device__ inline void result_pieces(const f32x16 &x, int kq, float scale, h8 &h, h8 &l)
{
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = x[8 * kq + j] * scale;
    split8(v, h, l);
}
// a tile of X: [rows / 32][half], both numbers
struct Pieces {
    h8 h[2][2], l[2][2];
};
__device__ inline int result_row(int e, int lane) { return 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3); }
__device__ inline f32x16 mfma3(const h8 &ah, const h8 &al, const h8 &bh, const h8 &bl, f32x16 c)
{
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, bh, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bl, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bh, c, 0, 0, 0);
}
// P times a tile of X, scaled twice; ACROSS: transposed
template <bool ACROSS> __device__ inline void tile_product(const Pieces &x, const h8 (*pf)[2][2][2][64], int lane, f32x16 (&y)[2])
{
#pragma unroll
    for (int rb = 0; rb < 2; ++rb)
#pragma unroll
        for (int e = 0; e < 16; ++e) y[rb][e] = 0.f;
#pragma unroll
    for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int kq = 0; kq < 2; ++kq) {
            const h8 xh = x.h[mb][kq], xl = x.l[mb][kq];
            const h8 ph[2] = {pf[0][mb][kq][0][lane], pf[1][mb][kq][0][lane]}, pl[2] = {pf[0][mb][kq][1][lane], pf[1][mb][kq][1][lane]};
            // the two results in turn
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int rb = 0; rb < 2; ++rb) {
                    const h8 a = p == 0 ? xl : xh, b = p == 1 ? pl[rb] : ph[rb];
                    y[rb] = ACROSS ? __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, y[rb], 0, 0, 0) : __builtin_amdgcn_mfma_f32_32x32x16_f16(b, a, y[rb], 0, 0, 0);
                }
        }
}

// One value of a buffer at a lane's byte offset plus a uniform one; past the end: zero, or nothing stored.  The bounds check is one of the
// lane's offset; the uniform one has to lie inside the buffer by itself.
template <int DT> __device__ inline float buffer_get(__amdgpu_buffer_rsrc_t b, int lane_off, int off)
{
    if constexpr (DT == XCONV_F32) return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(b, lane_off, off, 0));
    else return st16_to_f32<DT>((uint16_t)__builtin_amdgcn_raw_buffer_load_b16(b, lane_off, off, 0));
}
template <int DT> __device__ inline void buffer_put(__amdgpu_buffer_rsrc_t b, int lane_off, int off, float v)
{
    if constexpr (DT == XCONV_F32) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), b, lane_off, off, 0);
    else if constexpr (DT == XCONV_BF16) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(short, (__bf16)v), b, lane_off, off, 0);
    else __builtin_amdgcn_raw_buffer_store_b16((short)f32_to_f16_rne(v), b, lane_off, off, 0);
}
constexpr int kNarrowOut = 0x40000000;      // a lane's offset of what does not exist

// GT, OT: types of G and of the result.  A call of a small matrix is latency, of the code's own fetching too: loads and stores are
// buffer instructions, whose bounds checks take the place of masks, and all loads go out before the first is waited for.
template <int GT, int OT, bool MUON> __global__ __launch_bounds__(kNarrowThreads, 2) void orth_narrow_kernel(NarrowList L)
{
    extern __shared__ char narrow_lds[];
    NarrowLds &S = *reinterpret_cast<NarrowLds *>(narrow_lds);
    const NarrowMat &q = L.mat[blockIdx.x];
    constexpr int GE = GT == XCONV_F32 ? 4 : 2, OE = OT == XCONV_F32 ? 4 : 2;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, hrow = 4 * (lane >> 5);
    const bool tall = q.rows > q.cols;
    const int m = tall ? q.cols : q.rows, n = tall ? q.rows : q.cols;
    const int rstride = tall ? 1 : q.cols, cstride = tall ? q.cols : 1, count = q.rows * q.cols;
    const auto G = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(q.G), 0, count * GE, 0x00020000);
    const auto M = __builtin_amdgcn_make_buffer_rsrc(q.M, 0, MUON ? count * 4 : 0, 0x00020000);
    const auto O = __builtin_amdgcn_make_buffer_rsrc(q.out, 0, count * OE, 0x00020000);
    // a wave's part of A and P between the products: rows 32 mb + 16 kq .. of columns 32 rb ..
    const int rb0 = wave >> 2, mb0 = (wave >> 1) & 1, kq0 = wave & 1;
    // register e of rows 32 mb .. lies a multiple of the rows' distance, the same for all lanes, behind the lane's own place
    auto row_of = [](int mb, int e) { return 32 * mb + 8 * (e >> 2) + (e & 3); };
    auto first_of = [&](int i) { return 32 * (wave + kNarrowWaves * i); };
    f32x16 u[kNarrowTiles][2], mo[MUON ? kNarrowTiles : 1][2];
#pragma unroll
    for (int i = 0; i < kNarrowTiles; ++i) {
        if (first_of(i) >= n) continue;
        const int col = first_of(i) + c, place = col < n ? hrow * rstride + col * cstride : kNarrowOut / 4;
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int at = hrow + row_of(mb, e) < m ? place : kNarrowOut / 4, off = min(row_of(mb, e), m - 1) * rstride;
                u[i][mb][e] = buffer_get<GT>(G, at * GE, off * GE);
                if constexpr (MUON) mo[i][mb][e] = buffer_get<XCONV_F32>(M, at * 4, off * 4);
            }
    }
    double sq = 0.0;
#pragma unroll
    for (int i = 0; i < kNarrowTiles; ++i) {
        if (first_of(i) >= n) continue;
        const int col = first_of(i) + c, place = col < n ? hrow * rstride + col * cstride : kNarrowOut / 4;
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                if constexpr (MUON) {
                    const float g = u[i][mb][e], w = mo[i][mb][e] + (g - mo[i][mb][e]) * L.s.rest;
                    const int at = hrow + row_of(mb, e) < m ? place : kNarrowOut / 4, off = min(row_of(mb, e), m - 1) * rstride;
                    buffer_put<XCONV_F32>(M, at * 4, off * 4, w);
                    u[i][mb][e] = update_of(g, w, L.s);
                }
                sq += (double)u[i][mb][e] * u[i][mb][e];
            }
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) sq += __shfl_xor(sq, o);
    if (lane == 0) S.red[wave] = sq;
    {
        // P = I for the first X X^T, which needs X the other way round only
        h8 one, none;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            one[j] = (_Float16)(32 * mb0 + 16 * kq0 + result_row(j, lane) == 32 * rb0 + c ? kOrthScale : 0.f);
            none[j] = (_Float16)0.f;
        }
        S.pf[rb0][mb0][kq0][0][lane] = one;
        S.pf[rb0][mb0][kq0][1][lane] = none;
    }
    __syncthreads();
    sq = 0.0;
#pragma unroll
    for (int w = 0; w < kNarrowWaves; ++w) sq += S.red[w];
    const double norm = sqrt(sq), d = norm < (double)L.s.eps ? (double)L.s.eps : norm;      // (a NaN stays one)
    // 4096 / d in two factors, the first a power of two: a norm far from one takes a single float out of its range
    const int power = d > 0.0 && d < 1e300 ? max(-126, min(126, -ilogb(d))) : 0;
    const float s1 = ldexpf(1.f, power), s2 = d == 0.0 ? 0.f : (float)((double)kOrthScale / d / (double)s1);      // (eps = 0 and a zero matrix)
    Pieces x[kNarrowTiles];
#pragma unroll
    for (int i = 0; i < kNarrowTiles; ++i) {
        if (first_of(i) >= n) continue;
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
            for (int kq = 0; kq < 2; ++kq) {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = u[i][mb][8 * kq + j] * s1 * s2;
                split8(v, x[i].h[mb][kq], x[i].l[mb][kq]);
            }
    }
    __syncthreads();     // (the sums of squares lie where X X^T goes)

    for (int step = 0; step < L.steps; ++step) {
        // X <- P X, and the wave's part of X X^T
        f32x16 g[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 16; ++e) g[k][e] = 0.f;
#pragma unroll
        for (int i = 0; i < kNarrowTiles; ++i) {
            if (32 * (wave + kNarrowWaves * i) >= n) continue;
            // transposed first, for X X^T: one product's sums are live at a time
            {
                f32x16 z[2];
                tile_product<true>(x[i], S.pf, lane, z);
#pragma unroll
                for (int kq = 0; kq < 2; ++kq) {
                    h8 h[2], l[2];
#pragma unroll
                    for (int rb = 0; rb < 2; ++rb) result_pieces(z[rb], kq, 1.f / kOrthScale, h[rb], l[rb]);
#pragma unroll
                    for (int p = 0; p < 3; ++p)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            g[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p == 0 ? l[k >> 1] : h[k >> 1], p == 1 ? l[k & 1] : h[k & 1], g[k], 0, 0, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (step > 0) {
                f32x16 y[2];
                tile_product<false>(x[i], S.pf, lane, y);
#pragma unroll
                for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                    for (int kq = 0; kq < 2; ++kq) result_pieces(y[rb], kq, 1.f / kOrthScale, x[i].h[rb][kq], x[i].l[rb][kq]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) S.gram[wave][k][e][lane] = f32x4{g[k][4 * e], g[k][4 * e + 1], g[k][4 * e + 2], g[k][4 * e + 3]};
        __syncthreads();
        // The wave's part of A, added up in order of the waves: eight registers of a block, which are a fragment of A as an
        // operand as well (A is symmetric)
        float part[8], v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) part[j] = 0.f;
#pragma unroll
        for (int w = 0; w < kNarrowWaves; ++w)
#pragma unroll
            for (int j = 0; j < 8; j += 4) {
                const f32x4 t = S.gram[w][2 * mb0 + rb0][2 * kq0 + j / 4][lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) part[j + i] += t[i];
            }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            part[j] *= kOrthUnscale;
            v[j] = part[j] * kOrthScale;
        }
        split8(v, S.af[rb0][mb0][kq0][0][lane], S.af[rb0][mb0][kq0][1][lane]);
        __syncthreads();
        // the same part of P = a I + b A + c A A (two waves make a block of A A, each takes its half)
        f32x16 t;
#pragma unroll
        for (int e = 0; e < 16; ++e) t[e] = 0.f;
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
            for (int kq = 0; kq < 2; ++kq)
                t = mfma3(S.af[mb0][mb][kq][0][lane], S.af[mb0][mb][kq][1][lane], S.af[rb0][mb][kq][0][lane], S.af[rb0][mb][kq][1][lane], t);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float square = (kq0 ? t[8 + j] : t[j]) * kOrthUnscale;
            v[j] = L.s.b * part[j] + L.s.c * square;
            if (32 * mb0 + 16 * kq0 + result_row(j, lane) == 32 * rb0 + c) v[j] += L.s.a;
            v[j] *= kOrthScale;
        }
        split8(v, S.pf[rb0][mb0][kq0][0][lane], S.pf[rb0][mb0][kq0][1][lane]);
        __syncthreads();
    }

    // the last P X, along the rows of the result; no step: X_0
    const bool across = tall && L.steps > 0;
#pragma unroll
    for (int i = 0; i < kNarrowTiles; ++i) {
        const int n0 = first_of(i);
        if (n0 >= n) continue;
        // registers run along the rows from the lane's column, or (across) along the columns from the lane's row
        const int stride = across ? cstride : rstride, most = (across ? n - n0 : m) - hrow;
        int place[2], next[2];
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
            place[rb] = across ? (32 * rb + c) * rstride + (n0 + hrow) * cstride : hrow * rstride + (n0 + c) * cstride;
            next[rb] = across ? 0 : 32 * rb;
            if (across ? 32 * rb + c >= m : n0 + c >= n) place[rb] = kNarrowOut / 4;
        }
        auto at = [&](int rb, int e) { return next[rb] + row_of(0, e) < most ? place[rb] : kNarrowOut / 4; };
        const int end = (across ? n - n0 : m) - 1;
        auto along = [&](int rb, int e) { return min(next[rb] + row_of(0, e), end) * stride * OE; };
        f32x16 w[2], y[2];
        if constexpr (MUON) {
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                for (int e = 0; e < 16; ++e) w[rb][e] = buffer_get<OT>(O, at(rb, e) * OE, along(rb, e));
        }
        if (across) {
            tile_product<true>(x[i], S.pf, lane, y);
        } else if (L.steps > 0) {
            tile_product<false>(x[i], S.pf, lane, y);
        } else {
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                for (int e = 0; e < 16; ++e) y[rb][e] = ((float)x[i].h[rb][e >> 3][e & 7] + (float)x[i].l[rb][e >> 3][e & 7]) * kOrthScale;
        }
#pragma unroll
        for (int rb = 0; rb < 2; ++rb)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float o = y[rb][e] * kOrthUnscale;
                buffer_put<OT>(O, at(rb, e) * OE, along(rb, e), MUON ? w[rb][e] * L.s.keep - q.wscale * o : o);
            }
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Tiles of 128 x 128 read half as much for the same products, tiles of 64 x 64 waste less of a small matrix and are four times
// as many.  A product is taken in tiles of 128 where that leaves enough workgroups for the chip's 256 compute units (8 of 512 x 4608:
// X X^T 43 us in tiles of 128 and 62 us in tiles of 64; A A, which has 80 tiles of 128 there, 43 and 17 us).
//
// Sums along k are split so that a matrix has about as many workgroups as the chip has compute units, or twice as many of the
// large tiles: by the matrix' own extents, so that what else is in the call does not change its result.  A run of fewer than 24 (large
// tiles: 40) blocks costs more in the launch that joins than it gives.  Products of square matrices are split from 1536 rows on
// (five steps of 2048 x 4096: 1022 us with three runs, 1203 with one; 1024 x 2048: 364 us with two runs, 311 with one).
int splits_of(int m, int kblocks)
{
    const int t64 = ceil_div(m, 64) * (ceil_div(m, 64) + 1) / 2, t128 = ceil_div(m, 128) * (ceil_div(m, 128) + 1) / 2;
    const int want = m <= 1024 ? (224 + t64 / 2) / t64 : 448 / t128;
    return std::max(1, std::min(want, kblocks / (m <= 1024 ? 24 : 40)));
}
bool narrow(const xconv_orth_item &it) { return std::min(it.rows, it.cols) <= kNarrowM && std::max(it.rows, it.cols) <= kNarrowN; }

constexpr int kMergeM = 256;        // most rows of a matrix that takes both products by A in one launch

// Steps on A alone.  A step's polynomial P of A commutes with A, so the next step's A is P A P and two steps are one product
// P' P by X: three products of m x m matrices take the place of X X^T and P X.  That is less work where n > m, but more launches: a
// matrix alone gains from about 700000 values on (five steps, one at a time against groups: 512 x 4608 238 and 210 us, 512 x 1024 176
// and 187, 256 x 2304 137 and 147), several at once earlier (8 of 512 x 4608 820 and 530, 8 of 512 x 1024 335 and 313, 6 of 256 x 2304
// 209 and 181, 16 of 256 x 1152 293 and 193).  Less wide matrices gain too little (4 of 700 x 1100 358 and 350).  The rule cannot look at the
// rest of a call, which would change a result's bits: a single matrix between the two sizes pays for it.
bool grouped(const xconv_orth_item &it)
{
    const int m = std::min(it.rows, it.cols), n = std::max(it.rows, it.cols);
    return m >= 128 && n >= 2 * m && (long long)m * n >= 1 << 18;
}
// The steps in groups of at most three, then two.  An error of A is multiplied by up to |d (l q(l)^2) / dl| a step (l: an eigenvalue
// of A, q the polynomial), 11.9 with a = 3.44, where it would fade with a new X X^T; at the start A is small.  Products of P are kept as
// a sixteenth of themselves, below 16.  Five steps with a = 3.44, simulated: gradients of 200 to 800 rows 2.2e-6 to 3.2e-6 in groups of
// three and two, 1.3e-6 to 2.3e-6 one at a time and with fp32 products; matrices of equal singular values 2.7e-6 to 7.4e-6 against
// 1.5e-6 to 2.1e-6; one large singular value above equal ones 2.3e-5 against 9e-6, a dominant column 6e-6 against 8e-7, 384 x 900; below
// 128 rows up to 1e-5 against 1.3e-6.
int groups_of(const xconv_orth_args *args, int (&sizes)[64])
{
    int groups = 0;
    double top = 1.0;
    for (int k = 0; k < args->steps;) {
        const int most = k == 0 ? 3 : 2;
        double growth = 1.0, largest = 1.0;
        int n = 0;
        for (; n < most && k < args->steps; ++n, ++k) {
            double g = 0.0, p = 0.0, next = 0.0;
            for (int j = 0; j <= 512; ++j) {
                const double v = top * j / 512, l = v * v, q = args->a + (args->b + args->c * l) * l, slope = args->b + 2.0 * args->c * l;
                g = std::max(g, std::fabs(q * q + 2.0 * l * q * slope));
                p = std::max(p, std::fabs(q));
                next = std::max(next, std::fabs(v * q));
            }
            if (n > 0 && (growth > 160.0 || largest * p > 192.0)) break;
            growth *= std::max(1.0, g);
            largest *= p;
            top = next;
        }
        sizes[groups++] = n;
    }
    return groups;
}
constexpr float kGroupScale = 1.f / 16.f;
struct OrthPlan {
    int count, merge_mb, merge_cb;  // blocks of 32 rows and columns of the workgroups of that launch
    struct Mat {
        int m, n, mp, np, big[3], merge, squares, gsplits, gkbs, psplits, pkbs, tiles[3];
        size_t x, a, part, bytes;
    } mat[kOrthItems];
    size_t bytes;
};
// items: the matrices of a run, all of them wide
OrthPlan plan_orth(const xconv_orth_item *const *items, int count)
{
    OrthPlan P{};
    P.count = count;
    auto can = [](int m) { return m > kMergeM; };
    auto runs = [](int m, int n) { return splits_of(m, round_up(n, 64) / 16); };              // of X X^T
    auto runs_square = [&](int m) { return m <= 1536 ? 1 : runs(m, m); };                    // of the others
    long long large[3] = {0, 0, 0};     // workgroups with tiles of 128
    for (int i = 0; i < count; ++i) {
        const int m = std::min(items[i]->rows, items[i]->cols), n = std::max(items[i]->rows, items[i]->cols), tm = ceil_div(m, 128);
        if (!can(m)) continue;
        large[0] += (long long)tm * (tm + 1) / 2 * runs(m, n);
        large[1] += (long long)tm * (tm + 1) / 2 * runs_square(m);
        large[2] += (long long)tm * ceil_div(n, 128);
    }
    long long columns = 0;
    P.bytes = up256(sizeof(OrthMat) * kOrthItems);
    for (int i = 0; i < count; ++i) {
        OrthPlan::Mat &q = P.mat[i];
        q.m = std::min(items[i]->rows, items[i]->cols);
        q.n = std::max(items[i]->rows, items[i]->cols);
        int T = 64;
        for (int k = 0; k < 3; ++k) {
            q.big[k] = can(q.m) && large[k] >= 256;
            if (q.big[k]) T = 128;
        }
        q.mp = round_up(q.m, T);
        q.np = round_up(q.n, T);
        q.merge = q.m <= kMergeM && !grouped(*items[i]);
        if (q.merge) {
            P.merge_mb = std::max(P.merge_mb, q.mp <= 128 ? 4 : 8);
            columns += q.np;
        }
        for (int k = 0; k < 3; ++k) {
            const int t = q.big[k] ? 128 : 64;
            q.tiles[k] = k < 2 ? q.mp / t * (q.mp / t + 1) / 2 : q.mp / t * (q.np / t);
        }
        // (extents padded to 64 for the splits, runs of whole steps)
        auto split = [&](int extent, int &count, int &run) {
            const int kb = round_up(extent, 64) / 16;
            run = count > 1 ? round_up(ceil_div(kb, count), 4) : std::max(q.mp, q.np) / 16;
            if (count > 1) count = ceil_div(kb, run);
        };
        q.gsplits = runs(q.m, q.n);
        q.psplits = runs_square(q.m);
        split(q.n, q.gsplits, q.gkbs);
        split(q.m, q.psplits, q.pkbs);
        q.x = up256((size_t)q.mp * q.np * 4);
        q.a = (size_t)q.mp * q.mp * 4;       // (a multiple of 256)
        auto partial = [&](int k, int count) { return count > 1 ? (size_t)q.tiles[k] * count * (q.big[k] ? 128 * 128 : 64 * 64) * 4 : 0; };
        q.part = up256(std::max(partial(0, q.gsplits), partial(1, q.psplits)));
        q.squares = grouped(*items[i]) ? 4 : q.merge ? 1 : 2;
        q.bytes = 3 * q.x + q.squares * q.a + q.part + up256(kOrthNorms * sizeof(double));
        P.bytes += q.bytes;
    }
    // (64 columns read A half as often; 32 are twice as many workgroups)
    P.merge_cb = columns / 64 >= 192 ? 2 : 1;
    return P;
}

}  // namespace

namespace {
// What a matrix takes: one workgroup, a step at a time, steps in groups
enum { NARROW, SINGLE, GROUPED };
int kind_of(const xconv_orth_item &it) { return narrow(it) ? NARROW : grouped(it) ? GROUPED : SINGLE; }

// Calls `run` with the next kOrthItems matrices of a kind until there are none.  Within a run those of few rows come first: their
// workgroups make room early for the last ones of a launch that has a few more than the chip holds.
template <class F> bool wide_runs(const xconv_orth_item *items, int count, int kind, F &&run)
{
    const xconv_orth_item *list[kOrthItems];
    int n = 0;
    for (int i = 0; i <= count; ++i) {
        if (i < count && kind_of(items[i]) == kind) list[n++] = items + i;
        if (n == kOrthItems || (i == count && n)) {
            std::stable_sort(list, list + n, [](const xconv_orth_item *a, const xconv_orth_item *b) { return std::min(a->rows, a->cols) < std::min(b->rows, b->cols); });
            if (!run(list, n)) return false;
            n = 0;
        }
    }
    return true;
}
// the scratch of the runs of a kind, which go one after the other through it
size_t kind_ws(const xconv_orth_item *items, int count, int kind)
{
    size_t most = 0;
    wide_runs(items, count, kind, [&](const xconv_orth_item *const *list, int n) {
        most = std::max(most, plan_orth(list, n).bytes);
        return true;
    });
    return most;
}

OrthScalars scalars_of(const xconv_orth_args *args, const xconv_muon_args64 *muon)
{
    OrthScalars s{};
    s.g_dtype = args->g_dtype; s.out_dtype = args->out_dtype;
    s.a = args->a; s.b = args->b; s.c = args->c; s.eps = args->eps;
    if (muon) {
        s.muon = 1; s.nesterov = muon->nesterov != 0; s.mu = (float)muon->momentum;
        s.rest = (float)(1.0 - muon->momentum);
        s.keep = (float)(1.0 - muon->lr * muon->weight_decay);
    }
    return s;
}
float wscale_of(const xconv_orth_item &it, const xconv_muon_args64 *muon)
{
    return muon ? (float)(muon->lr * std::sqrt(std::max(1.0, (double)it.rows / it.cols))) : 0.f;
}

hipError_t launch_narrow(const xconv_orth_item *items, int count, const xconv_orth_args *args, const xconv_muon_args64 *muon, hipStream_t st)
{
    typedef void (*Kernel)(NarrowList);
    // [muon][type of G][type of the result]
    static const Kernel kernels[2][3][3] = {
        {{orth_narrow_kernel<0, 0, false>, orth_narrow_kernel<0, 1, false>, orth_narrow_kernel<0, 2, false>},
         {orth_narrow_kernel<1, 0, false>, orth_narrow_kernel<1, 1, false>, orth_narrow_kernel<1, 2, false>},
         {orth_narrow_kernel<2, 0, false>, orth_narrow_kernel<2, 1, false>, orth_narrow_kernel<2, 2, false>}},
        {{orth_narrow_kernel<0, 0, true>, orth_narrow_kernel<0, 1, true>, orth_narrow_kernel<0, 2, true>},
         {orth_narrow_kernel<1, 0, true>, orth_narrow_kernel<1, 1, true>, orth_narrow_kernel<1, 2, true>},
         {orth_narrow_kernel<2, 0, true>, orth_narrow_kernel<2, 1, true>, orth_narrow_kernel<2, 2, true>}}};
    static const hipError_t set = [] {
        hipError_t e = hipSuccess;
        for (const Kernel *k1 = &kernels[0][0][0]; k1 < &kernels[0][0][0] + 18; ++k1)
            if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void *>(*k1), hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(NarrowLds));
        return e;
    }();
    if (set != hipSuccess) return set;
    const Kernel kernel = kernels[muon != nullptr][args->g_dtype][args->out_dtype];
    NarrowList L{};
    L.s = scalars_of(args, muon);
    L.steps = args->steps;
    int n = 0;
    for (int i = 0; i <= count; ++i) {
        if (i < count && narrow(items[i])) {
            const xconv_orth_item &it = items[i];
            L.mat[n++] = {it.G_dev, it.out_dev, it.M_dev, it.rows, it.cols, wscale_of(it, muon)};
        }
        if (n == kNarrowItems || (i == count && n)) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(kNarrowThreads), sizeof(NarrowLds), st, L);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            n = 0;
        }
    }
    return hipSuccess;
}

template <int MB, int CB> hipError_t allow_merge()
{
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(orth_merge_kernel<MB, CB, 0>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(MergeLds<MB, CB>));
    return e != hipSuccess ? e : hipFuncSetAttribute(reinterpret_cast<const void *>(orth_merge_kernel<MB, CB, 1>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(MergeLds<MB, CB>));
}
template <int MB, int CB> void launch_merge(const OrthRef &R, int odd, bool last, hipStream_t st)
{
    const dim3 grid((unsigned)R.total), block(64 * MB);
    if (last) hipLaunchKernelGGL((orth_merge_kernel<MB, CB, 1>), grid, block, sizeof(MergeLds<MB, CB>), st, R, odd);
    else hipLaunchKernelGGL((orth_merge_kernel<MB, CB, 0>), grid, block, sizeof(MergeLds<MB, CB>), st, R, odd);
}

hipError_t launch_wide(const xconv_orth_item *const *items, int count, const xconv_orth_args *args, const xconv_muon_args64 *muon, void *ws, hipStream_t st)
{
    static const hipError_t set = allow_merge<8, 2>();      // (the others stay below 64 KB)
    if (set != hipSuccess) return set;
    const OrthPlan P = plan_orth(items, count);
    OrthList L{};
    L.s = scalars_of(args, muon);
    L.s.count = count;
    char *p = static_cast<char *>(ws);
    auto take = [&](size_t bytes) { char *r = p; p += bytes; return r; };
    OrthMat *list = (OrthMat *)take(up256(sizeof(OrthMat) * kOrthItems));
    // the first workgroups of the matrices in the launches (products: tiles of 64, of 128)
    enum { NORM, START, XX, XX_JOIN = XX + 2, SQUARE, SQUARE_JOIN = SQUARE + 2, APPLY, MERGE = APPLY + 2, KINDS };
    OrthRef R[KINDS];
    for (OrthRef &r : R) r = OrthRef{L.s, 0, {}, list, {}};
    for (int i = 0; i < count; ++i) {
        const xconv_orth_item &it = *items[i];
        const OrthPlan::Mat &f = P.mat[i];
        OrthMat &q = L.mat[i];
        q.G = it.G_dev; q.out = it.out_dev; q.M = it.M_dev;
        q.rows = it.rows; q.cols = it.cols; q.m = f.m; q.n = f.n; q.mp = f.mp; q.np = f.np;
        for (int k = 0; k < 3; ++k) q.big[k] = f.big[k];
        q.gsplits = f.gsplits; q.gkbs = f.gkbs; q.psplits = f.psplits; q.pkbs = f.pkbs;
        q.X = (_Float16 *)take(f.x); q.Xt = (_Float16 *)take(f.x); q.Xt2 = (_Float16 *)take(f.x);
        q.S = (_Float16 *)take(f.squares * f.a);
        q.part = (float *)take(f.part);
        q.sq = (double *)take(up256(kOrthNorms * sizeof(double)));
        q.nsq = (int)std::min<size_t>(kOrthNorms, ((size_t)it.rows * it.cols + 4095) / 4096);
        q.wscale = wscale_of(it, muon);
        int blocks[KINDS] = {};
        blocks[NORM] = q.nsq;
        blocks[START] = (f.mp / kOrthTile) * (f.np / kOrthTile);
        blocks[XX + f.big[0]] = f.tiles[0] * f.gsplits;
        blocks[XX_JOIN] = f.gsplits > 1 ? f.tiles[0] * (f.big[0] ? 4 : 1) : 0;
        if (f.merge) blocks[MERGE] = f.np / (32 * P.merge_cb);
        else blocks[SQUARE + f.big[1]] = f.tiles[1] * f.psplits;
        blocks[SQUARE_JOIN] = !f.merge && f.psplits > 1 ? f.tiles[1] * (f.big[1] ? 4 : 1) : 0;
        if (!f.merge) blocks[APPLY + f.big[2]] = f.tiles[2];
        for (int k = 0; k < KINDS; ++k) {
            R[k].first[i] = R[k].total;
            R[k].total += blocks[k];
        }
    }
    for (int i = 0; i < count; ++i) L.first[i] = R[NORM].first[i];
    for (OrthRef &r : R) r.one = L.mat[0];
    const dim3 block(kThreads);
    // (products: whole rounds of the eight dies)
    auto go = [&](auto kernel, int k, auto... more) {
        if (!R[k].total) return;
        const int blocks = (k >= XX && k < XX_JOIN) || (k >= SQUARE && k < SQUARE_JOIN) || (k >= APPLY && k < MERGE) ? round_up(R[k].total, 8) : R[k].total;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), block, 0, st, R[k], more...);
    };
    hipLaunchKernelGGL(orth_norm_kernel, dim3((unsigned)R[NORM].total), block, 0, st, L, list);
    go(orth_start_kernel, START);
    if (args->steps == 0) go(orth_none_kernel, START);
    // S_out = polynomial of A, or S_left S_right
    auto poly = [&](int out) {
        const Squares u{0, 0, out, 1.f};
        go(orth_square_kernel<64, POLY>, SQUARE, u);
        go(orth_square_kernel<128, POLY>, SQUARE + 1, u);
        go(orth_join_kernel<POLY>, SQUARE_JOIN, u);
    };
    auto mul = [&](int left, int right, int out, float scale = 1.f) {
        const Squares u{left, right, out, scale};
        go(orth_square_kernel<64, MUL>, SQUARE, u);
        go(orth_square_kernel<128, MUL>, SQUARE + 1, u);
        go(orth_join_kernel<MUL>, SQUARE_JOIN, u);
    };
    int sizes[64], groups = args->steps;
    if (grouped(*items[0])) groups = groups_of(args, sizes);
    else std::fill(sizes, sizes + groups, 1);
    for (int k = 0; k < groups; ++k) {
        const int odd = k & 1;
        const bool last = k + 1 == groups;
        const Squares gram{0, 0, 0, 1.f};
        go(orth_square_kernel<64, GRAM>, XX, gram);
        go(orth_square_kernel<128, GRAM>, XX + 1, gram);
        go(orth_join_kernel<GRAM>, XX_JOIN, gram);
        // A is S_0, the last polynomial S_p, the product of all of the group S_q, and S_t is free
        int p = 1, q = 1, t = 2;
        poly(p);
        for (int j = 1; j < sizes[k]; ++j) {
            mul(0, p, t);
            mul(t, p, 0);
            poly(t);
            const int out = j == 1 ? 3 : p, free = j == 1 ? p : q;
            mul(t, q, out, j == 1 ? kGroupScale : 1.f);
            p = t;
            q = out;
            t = free;
        }
        const float scale = sizes[k] > 1 ? 1.f / kGroupScale : 1.f;
        if (R[MERGE].total) {
            if (P.merge_mb == 4 && P.merge_cb == 1) launch_merge<4, 1>(R[MERGE], odd, last, st);
            else if (P.merge_mb == 4) launch_merge<4, 2>(R[MERGE], odd, last, st);
            else if (P.merge_cb == 1) launch_merge<8, 1>(R[MERGE], odd, last, st);
            else launch_merge<8, 2>(R[MERGE], odd, last, st);
        }
        if (!last) {
            go(orth_apply_kernel<64, 0>, APPLY, odd, q, scale);
            go(orth_apply_kernel<128, 0>, APPLY + 1, odd, q, scale);
        } else {
            go(orth_apply_kernel<64, 1>, APPLY, odd, q, scale);
            go(orth_apply_kernel<128, 1>, APPLY + 1, odd, q, scale);
        }
    }
    return hipGetLastError();
}
}  // namespace

namespace {
// Streams beside the caller's for the kinds of matrices of a call: each kind is a chain of launches that leave most of the chip idle
// (18 layers of three kinds: 379 us one kind after the other, 215 us beside each other, with 11 bits in the last product; 64 x 576 and 128 x 1152: 146 and 111).  They start after what the caller's stream holds
// and it goes on after them, so a call looks as if all of it ran there.  Kept for later calls; one call at a time has them.
struct Sides {
    int device;
    hipStream_t stream[2];
    hipEvent_t start, done[2];
    Sides *next;
};
std::mutex g_sides_mu;
Sides *g_sides = nullptr;       // those that no call has; a list that takes no memory to put one back (never destroyed: the runtime may be gone by then)
// null: none to be had
Sides *take_sides()
{
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) return nullptr;
    {
        std::lock_guard<std::mutex> lk(g_sides_mu);
        for (Sides **p = &g_sides; *p; p = &(*p)->next)
            if ((*p)->device == device) {
                Sides *s = *p;
                *p = s->next;
                return s;
            }
    }
    Sides *s = new (std::nothrow) Sides{device, {nullptr, nullptr}, nullptr, {nullptr, nullptr}, nullptr};
    if (!s) return nullptr;
    bool ok = hipEventCreateWithFlags(&s->start, hipEventDisableTiming) == hipSuccess;
    for (int i = 0; i < 2; ++i)
        ok = ok && hipStreamCreateWithFlags(&s->stream[i], hipStreamNonBlocking) == hipSuccess && hipEventCreateWithFlags(&s->done[i], hipEventDisableTiming) == hipSuccess;
    if (ok) return s;
    for (int i = 0; i < 2; ++i) {
        if (s->done[i]) (void)hipEventDestroy(s->done[i]);
        if (s->stream[i]) (void)hipStreamDestroy(s->stream[i]);
    }
    if (s->start) (void)hipEventDestroy(s->start);
    delete s;
    return nullptr;
}
void give_sides(Sides *s)
{
    std::lock_guard<std::mutex> lk(g_sides_mu);
    s->next = g_sides;
    g_sides = s;
}
}  // namespace

size_t orth_ws_bytes(const xconv_orth_item *items, int count)
{
    return std::max<size_t>(256, kind_ws(items, count, SINGLE) + kind_ws(items, count, GROUPED));
}

void orth_plan_info(const xconv_orth_item *items, int count, const xconv_orth_args *args, int index, int32_t *out)
{
    std::fill(out, out + 16, 0);
    const xconv_orth_item *it = items + index;
    const int kind = kind_of(*it);
    out[0] = kind;
    int sizes[64], groups = args->steps;
    std::fill(sizes, sizes + groups, 1);
    if (kind == GROUPED) groups = groups_of(args, sizes);
    out[8] = groups;
    for (int k = 0; k < std::min(groups, 7); ++k) out[9 + k] = sizes[k];
    if (kind == NARROW) return;
    wide_runs(items, count, kind, [&](const xconv_orth_item *const *list, int n) {
        const int at = (int)(std::find(list, list + n, it) - list);
        if (at == n) return true;
        const OrthPlan P = plan_orth(list, n);
        const OrthPlan::Mat &q = P.mat[at];
        for (int k = 0; k < 3; ++k) out[1 + k] = k > 0 && q.merge ? 0 : q.big[k] ? 128 : 64;
        out[4] = q.gsplits;
        out[5] = q.merge ? 0 : q.psplits;
        if (q.merge) {
            out[6] = 32 * P.merge_mb;
            out[7] = 32 * P.merge_cb;
        }
        return false;
    });
}

hipError_t launch_orth(const xconv_orth_item *items, int count, const xconv_orth_args *args, const xconv_muon_args64 *muon, void *ws, hipStream_t st)
{
    bool any[3] = {};
    for (int i = 0; i < count; ++i) any[kind_of(items[i])] = true;
    auto run = [&](int kind, hipStream_t on) {
        if (kind == NARROW) return launch_narrow(items, count, args, muon, on);
        void *at = kind == GROUPED ? static_cast<char *>(ws) + kind_ws(items, count, SINGLE) : ws;
        hipError_t e = hipSuccess;
        wide_runs(items, count, kind, [&](const xconv_orth_item *const *list, int n) { return (e = launch_wide(list, n, args, muon, at, on)) == hipSuccess; });
        return e;
    };
    // (not while the caller's stream is captured: streams of a capture are not to be used by other calls until its end)
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    Sides *sides = nullptr;
    if (any[NARROW] + any[SINGLE] + any[GROUPED] > 1) {
        if (hipStreamIsCapturing(st, &capture) == hipSuccess && capture == hipStreamCaptureStatusNone) sides = take_sides();
        if (!sides) (void)hipGetLastError();
    }
    hipError_t e = hipSuccess;
    if (!sides) {
        for (int kind : {NARROW, GROUPED, SINGLE})
            if (any[kind] && e == hipSuccess) e = run(kind, st);
        return e;
    }
    // the longest chain stays on the caller's stream
    const int own = any[GROUPED] ? GROUPED : SINGLE;
    int used = 0;
    e = hipEventRecord(sides->start, st);
    for (int kind : {NARROW, GROUPED, SINGLE}) {
        if (!any[kind] || e != hipSuccess) continue;
        hipStream_t on = st;
        if (kind != own) {
            on = sides->stream[used];
            e = hipStreamWaitEvent(on, sides->start, 0);
            if (e != hipSuccess) break;
            ++used;
        }
        e = run(kind, on);
    }
    // also after an error: what was launched ends before the caller's stream goes on
    for (int i = 0; i < used; ++i) {
        hipError_t j = hipEventRecord(sides->done[i], sides->stream[i]);
        if (j == hipSuccess) j = hipStreamWaitEvent(st, sides->done[i], 0);
        if (j != hipSuccess) (void)hipStreamSynchronize(sides->stream[i]);
        if (e == hipSuccess) e = j;
    }
    give_sides(sides);
    return e;
}

}  // namespace xc
