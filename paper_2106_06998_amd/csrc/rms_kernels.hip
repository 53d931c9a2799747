// Root-mean-square norm over the channels of every position, with the addition of a residual and the dropout in front of it.
//     forward   h = residual + drop(x), rstd = 1 / sqrt(sum_c h^2 / C + eps), y = h rstd gamma
//     8 bits    the same (no dropout), scale = max(max_c |y|, 2^-100) / top, q = y / scale rounded (top: 448 for e4m3, 127 for int8)
//     backward  g = dy gamma, xh = h rstd, dz = rstd (g - xh sum_c (g xh) / C) + dh, dresidual = dz, dx = drop(dz),
//               dgamma = sum over positions of dy xh
// Tensors are [outer, C, inner] as for layer normalisation (norm_core.h), which the division of the work follows too.  Bound by HBM:
// every tensor is read once; h stays in registers as floats, so that statistics and y are those of the unrounded sum, while the stored h
// is rounded once.  The mask of dropout is drawn in registers, in both passes.
//
// Backward: a workgroup walks positions and adds dgamma up in registers; the workgroups' sums are added in order by a second launch.
//
// Measured (three sets of tensors in turn): forward, 200704 rows of 128 bf16 with residual and dropout 35 us = 5.9 TB/s (205 MB, of which the
// 256 MB cache holds some); 8192 rows of 4096 fp16 26.8 us = 5.0 TB/s, the rate of a copy; 8 bits, 8192 rows of 5001 fp16 36.9 us = 3.3 TB/s
// (5000: 32; 8192: 47 = 4.2 TB/s); backward, 4096 rows of 4096 bf16 with the residual's gradient 31.8 us = 4.3 TB/s and 4.6 for the join of
// dgamma; 256 x 256 x 28 x 28 fp16 with residual and dropout 129 us = 4.0 TB/s (514 MB; 37 vector instructions a value, 13 of them for the
// mask, and the barrier between sums and outputs, which two workgroups a compute unit hide from each other only in part).
#include "drop.h"
#include "launch.h"
#include "norm_core.h"

namespace xc {

namespace {

struct RmsArgs : NormGeom {
    const void *x, *res, *gamma;  // forward: input and residual (or null); backward: x is the stored h
    const void *dy, *dh;          // backward; dh may be null
    void *y, *h;                  // forward: y or q, and h (null: not stored); backward: dresidual and dx (either may be null)
    float *rstd, *scale;          // rstd: written (forward, may be null) or read (backward); scale: of the 8-bit output
    float *part;                  // backward: [workgroups][C] partial sums of dgamma, null when it is not wanted
    DropArgs drop;
    float top;
    int w32, int8, fours;         // gamma in fp32; q is int8; dropout's places are multiples of 4
    int over;                     // an output lies over an input
};

// SHORT: vectors may be shorter than V (rows shorter than a vector, and rows that are read again)
template <int DT, bool SHORT> __device__ inline uint4 get_part(const typename NormElem<DT>::t *run, const Part &p)
{
    if constexpr (SHORT) return load_part<DT>(run, p);
    else return load_loose<DT>(run + p.at);
}
template <int DT, bool SHORT> __device__ inline void put_part(typename NormElem<DT>::t *run, const uint4 &v, const Part &p)
{
    if constexpr (SHORT) store_part<DT>(run, v, p);
    else store_loose<DT>(run + p.at, v);
}
// gamma's address anew: its values are loaded where they are used, not kept for the rows to come
__device__ inline const void *gamma_of(const RmsArgs &a)
{
    const void *p = a.gamma;
    asm volatile("" : "+s"(p));
    return p;
}
template <int DT, int V, bool SHORT> __device__ inline void load_gamma(const RmsArgs &a, const void *gamma, Part p, float (&g)[V])
{
    if constexpr (!SHORT) p.hi = V;
    if (DT == XCONV_F32 || a.w32) load_params<XCONV_F32, V>(gamma, p, 1.f, g);
    else load_params<DT, V>(gamma, p, 1.f, g);
}
template <int DT> __device__ inline float load_gamma1(const RmsArgs &a, int c)
{
    if (DT == XCONV_F32 || a.w32) return load_param<XCONV_F32>(a.gamma, c, 1.f);
    else return load_param<DT>(a.gamma, c, 1.f);
}

// ---- 8 bits --------------------------------------------------------------------------------------------------------
// The magnitude that a position's scale goes by; compared as bits, where a NaN is above everything and makes the scale a NaN
constexpr float kLeast8 = 0x1p-100f;
__device__ inline uint32_t magnitude(float y) { return __float_as_uint(y) & 0x7fffffffu; }

__device__ inline uint32_t four8(float a, float b, float c, float d, int int8)
{
    if (int8) {
        auto one = [](float v) { return (uint32_t)(int)fminf(fmaxf(rintf(v), -127.f), 127.f) & 0xffu; };
        // (a NaN would become -127 by fmaxf; it is 0, and the scale says NaN)
        auto safe = [&](float v) { return v == v ? one(v) : 0u; };
        return safe(a) | safe(b) << 8 | safe(c) << 16 | safe(d) << 24;
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);        // round to nearest even
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return (uint32_t)w;
}
// What h gamma is multiplied by: rstd ratio, ratio = top / max |y|.  Under a tiny eps that passes fp32 where y is zero or tiny (the least
// magnitude gives a ratio of 5.7e32, rstd may be 1e6 and more), and a zero would become a NaN: then (true) h gamma takes rstd first and f is
// the ratio, neither of which overflows.  One factor otherwise, at no cost: 8192 x 5001 fp16 36.4 us with and without the test.
__device__ inline bool factor8(float rstd, float ratio, float &f)
{
    f = rstd * ratio;
    const bool two = f == __builtin_inff() && rstd < __builtin_inff();
    f = two ? ratio : f;
    return two;
}
template <int V> struct __attribute__((packed, aligned(1))) Loose8 { uint32_t w[V / 4]; };
// V values from p.at on of the run
template <int V, bool SHORT> __device__ inline void store8(uint8_t *run, const Part &p, const float (&y)[V], int int8)
{
    Loose8<V> o;
#pragma unroll
    for (int j = 0; j < V / 4; ++j) o.w[j] = four8(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3], int8);
    if (!SHORT || p.hi == V) {
        *reinterpret_cast<Loose8<V> *>(run + p.at) = o;
    } else {
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
            if (i < p.hi) run[p.at + i] = (uint8_t)(o.w[i / 4] >> (8 * (i % 4)));
    }
}

// Largest of R values over a group of G lanes; for groups of several waves in two parts with a barrier of the caller's (group_sum's) between
// them: what a wave has, into `slot` of `red`, and what all have
template <int G, int R, int T> __device__ inline void group_max(uint32_t (&s)[R], uint32_t *red, int slot)
{
#pragma unroll
    for (int o = (G < 64 ? G : 64) / 2; o >= 1; o >>= 1)
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = max(s[r], (uint32_t)__shfl_xor((int)s[r], o));
    if (G > 64 && (threadIdx.x & 63) == 0)
#pragma unroll
        for (int r = 0; r < R; ++r) red[(slot * (T / 64) + (threadIdx.x >> 6)) * R + r] = s[r];
}
template <int G, int R, int T> __device__ inline void group_max_join(uint32_t (&s)[R], const uint32_t *red, int slot)
{
    if constexpr (G > 64) {
        const uint32_t *q = red + (slot * (T / 64) + (T > G ? threadIdx.x / G * (G / 64) : 0)) * R;
#pragma unroll
        for (int i = 0; i < G / 64; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r) s[r] = max(s[r], q[i * R + r]);
    }
}

// A thread's first vector (channel) anew: offsets and masks of its vectors are computed where they are used, not kept: the loop over the rows
// (tiles) would carry them along, for every vector more registers than its values take
__device__ inline int again(int first)
{
    asm volatile("" : "+v"(first));
    return first;
}

// ---- rows ----------------------------------------------------------------------------------------------------------
// Threads of a workgroup.  Groups of a wave and less wait for nobody; those of several waves are a workgroup of their own in the forward
// pass, so that a barrier holds up one row.
template <int G> constexpr int rms_fwd_threads = G > 64 ? G : 256;
// waves a SIMD that the forward pass leaves registers for: 8 registers a vector and lane hold h
template <int G, int K, int R> constexpr int rms_fwd_waves = K > 4 && G < 1024 ? 3 : K * R >= 4 ? 4 : K * R == 3 ? 5 : 6;

// G lanes a row, K vectors a lane, R rows at once; K == 0: a row is read again for its second pass.  OUT8: q and scale instead of y.
// One reduction a row: in the 8-bit form h becomes h gamma as soon as its square is in the sum, and the largest |h gamma| goes along (two
// reductions: 8192 x 8192 fp16 66 us, 47 so).
template <int DT, bool OUT8, int G, int K, int R>
__global__ __launch_bounds__(rms_fwd_threads<G>, (rms_fwd_waves<G, K, R>)) void rms_rows_fwd_kernel(RmsArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, T = rms_fwd_threads<G>, RP = T / G, KR = K > 0 ? K : 1;
    constexpr bool SHORT = G == 4 || K == 0, EARLY = OUT8;
    __shared__ float red[G > 64 ? 2 * R * (T / 64) : 1];
    __shared__ uint32_t redm[G > 64 && OUT8 ? 2 * R * (T / 64) : 1];
    int turn = 0;
    const int lane = threadIdx.x % G, grp = threadIdx.x / G;
    const int nv = (a.C + V - 1) / V;
    const elem_t *X = static_cast<const elem_t *>(a.x), *RES = static_cast<const elem_t *>(a.res);
    const bool drops = !OUT8 && a.drop.q16;
    const uint64_t key = drops ? drop_key(a.drop) : 0;
    auto rounds = [&](auto &&body) {
        if constexpr (K > 0) {
            const int l = again(lane);
#pragma unroll
            for (int k = 0; k < K; ++k) body(k, l + k * G);
        } else {
            for (int v = lane; v < nv; v += G) body(0, v);
        }
    };
    for (long long r0 = (long long)blockIdx.x * (RP * R); r0 < a.outer; r0 += (long long)gridDim.x * (RP * R)) {   // (the same count for all threads)
        const void *gamma = gamma_of(a);
        float h[R][KR][V];
        uint4 rx[R][KR], rr[R][KR];
        size_t at[R];
        bool on[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long row = r0 + r * RP + grp;
            on[r] = row < a.outer;
            at[r] = (size_t)(on[r] ? row : 0) * a.C;
        }
        auto get = [&](const elem_t *x, int r, int v, const Part &p) { return v < nv ? get_part<DT, SHORT>(x + at[r], p) : uint4{0, 0, 0, 0}; };
        auto make = [&](int r, int k, const Part &p) {
            unpack<DT>(rx[r][k], h[r][k]);
            if (drops) drop_values<V>(a.drop, key, at[r] + p.at, a.fours, h[r][k]);
            if (RES) {
                float t[V];
                unpack<DT>(rr[r][k], t);
#pragma unroll
                for (int i = 0; i < V; ++i) h[r][k][i] += t[i];
            }
        };
        if constexpr (K > 0) {
            rounds([&](int k, int v) {
                const Part p = part_of<V>(v, a.C, SHORT ? a.exact : 0);
#pragma unroll
                for (int r = 0; r < R; ++r) rx[r][k] = get(X, r, v, p);
            });
            if (RES)
                rounds([&](int k, int v) {
                    const Part p = part_of<V>(v, a.C, SHORT ? a.exact : 0);
#pragma unroll
                    for (int r = 0; r < R; ++r) rr[r][k] = get(RES, r, v, p);
                });
            // h may lie over what another lane's overlapping vector still reads
            if (a.over) {
                __builtin_amdgcn_s_waitcnt(0);
                if constexpr (G > 64) __syncthreads();
            }
        }
        float s[R];
        uint32_t m[R];
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = 0.f, m[r] = 0;
        rounds([&](int k, int v) {
            const Part p = part_of<V>(v, a.C, SHORT ? a.exact : 0);
            float g[V];
            if (EARLY) {
                if (v < nv) {
                    load_gamma<DT, V, SHORT>(a, gamma, p, g);
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) g[i] = 0.f;
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if constexpr (K == 0) {
                    rx[r][0] = get(X, r, v, p);
                    if (RES) rr[r][0] = get(RES, r, v, p);
                }
                make(r, k, p);
                if (K > 0 ? !masked<G>(a, k, nv) : !a.ragged) {
#pragma unroll
                    for (int i = 0; i < V; ++i) s[r] += h[r][k][i] * h[r][k][i];       // (zeros past the last vector)
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) s[r] += v < nv && own(p, i) ? h[r][k][i] * h[r][k][i] : 0.f;
                }
                if (K > 0 && a.h && on[r] && v < nv) put_part<DT, SHORT>(static_cast<elem_t *>(a.h) + at[r], pack<DT>(h[r][k]), p);
                if constexpr (EARLY) {
#pragma unroll
                    for (int i = 0; i < V; ++i) h[r][k][i] *= g[i];
#pragma unroll
                    for (int i = 0; i < V; ++i) m[r] = max(m[r], magnitude(h[r][k][i]));
                }
            }
        });
        const int slot = turn;
        if constexpr (OUT8) group_max<G, R, T>(m, redm, slot);
        group_sum<G, R, T>(s, red, turn);
        float rstd[R], f[R];
        bool two[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            rstd[r] = rstd_of(s[r], a);
            f[r] = rstd[r];
            two[r] = false;
        }
        if constexpr (OUT8) {
            group_max_join<G, R, T>(m, redm, slot);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float most = __uint_as_float(max(magnitude(__uint_as_float(m[r]) * rstd[r]), __float_as_uint(kLeast8)));
                two[r] = factor8(rstd[r], a.top / most, f[r]);
                if (lane == 0 && on[r]) a.scale[r0 + r * RP + grp] = most / a.top;
                if (K > 0 && two[r])
#pragma unroll
                    for (int k = 0; k < KR; ++k)
#pragma unroll
                        for (int i = 0; i < V; ++i) h[r][k][i] *= rstd[r];
            }
        }
        rounds([&](int k, int v) {
            if (v >= nv) return;
            const Part p = part_of<V>(v, a.C, SHORT ? a.exact : 0);
            float g[V];
            if (K == 0 || !EARLY) load_gamma<DT, V, SHORT>(a, gamma, p, g);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (!on[r]) continue;
                if constexpr (K == 0) {
                    rx[r][0] = get(X, r, v, p);
                    if (RES) rr[r][0] = get(RES, r, v, p);
                    make(r, 0, p);
                    if (a.h) put_part<DT, SHORT>(static_cast<elem_t *>(a.h) + at[r], pack<DT>(h[r][k]), p);
                }
                if constexpr (K == 0 && OUT8) {
#pragma unroll
                    for (int i = 0; i < V; ++i) h[r][k][i] = h[r][k][i] * g[i] * (two[r] ? rstd[r] : 1.f) * f[r];
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) h[r][k][i] *= EARLY ? f[r] : f[r] * g[i];
                }
                if constexpr (OUT8) store8<V, SHORT>(static_cast<uint8_t *>(a.y) + at[r], p, h[r][k], a.int8);
                else put_part<DT, SHORT>(static_cast<elem_t *>(a.y) + at[r], pack<DT>(h[r][k]), p);
            }
        });
        if (!OUT8 && lane == 0 && a.rstd) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (on[r]) a.rstd[r0 + r * RP + grp] = rstd[r];
        }
    }
}

// T threads, so T / G rows at once; every lane adds up dgamma of its own columns.  K == 0: one row a workgroup at a time, dgamma in the
// workgroup's own slots of `part`.
template <int DT, int G, int K, int R, int T>
__global__ __launch_bounds__(T, 4) void rms_rows_bwd_kernel(RmsArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, RP = T / G, KR = K > 0 ? K : 1;
    constexpr bool SHORT = G == 4 || K == 0;
    __shared__ float red[G > 64 ? 2 * R * (T / 64) : 1];
    int turn = 0;
    const int lane = threadIdx.x % G, grp = threadIdx.x / G;
    const elem_t *H = static_cast<const elem_t *>(a.x), *DY = static_cast<const elem_t *>(a.dy), *DH = static_cast<const elem_t *>(a.dh);
    elem_t *DR = static_cast<elem_t *>(a.y), *DX = static_cast<elem_t *>(a.h);
    const int nv = (a.C + V - 1) / V;
    const uint64_t key = a.drop.q16 ? drop_key(a.drop) : 0;
    float *part = a.part ? a.part + (size_t)blockIdx.x * a.C : nullptr;
    auto rounds = [&](auto &&body) {
        if constexpr (K > 0) {
            const int l = again(lane);
#pragma unroll
            for (int k = 0; k < K; ++k) body(k, l + k * G);
        } else {
            for (int v = lane; v < nv; v += G) body(0, v);
        }
    };
    float ag[KR][V];
#pragma unroll
    for (int k = 0; k < KR; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) ag[k][i] = 0.f;
    bool first = true;
    // what is read of R rows
    struct Rows {
        uint4 x[R][KR], d[R][KR], h[R][KR];
        float rstd[R];
    };
    auto fetch = [&](long long r0, Rows &f) {
        size_t at[R];
        bool on[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long row = r0 + r * RP + grp;
            on[r] = row < a.outer;
            at[r] = (size_t)(on[r] ? row : 0) * a.C;
            f.rstd[r] = on[r] ? a.rstd[row] : 0.f;
        }
        rounds([&](int k, int v) {
            const Part p = part_of<V>(v, a.C, SHORT ? a.exact : 0);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                f.x[r][k] = on[r] && v < nv ? get_part<DT, SHORT>(H + at[r], p) : uint4{0, 0, 0, 0};
                f.d[r][k] = on[r] && v < nv ? get_part<DT, SHORT>(DY + at[r], p) : uint4{0, 0, 0, 0};
            }
        });
        if (DH)
            rounds([&](int k, int v) {
                const Part p = part_of<V>(v, a.C, SHORT ? a.exact : 0);
#pragma unroll
                for (int r = 0; r < R; ++r) f.h[r][k] = on[r] && v < nv ? get_part<DT, SHORT>(DH + at[r], p) : uint4{0, 0, 0, 0};
            });
    };
    const long long step = (long long)gridDim.x * (RP * R);
    Rows next;
    if constexpr (K > 0) fetch((long long)blockIdx.x * (RP * R), next);
    for (long long r0 = (long long)blockIdx.x * (RP * R); r0 < a.outer; r0 += step, first = false) {   // (the same count for all threads)
        Rows now;
        float rstd[R], c[R];
        size_t at[R];
        bool on[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long row = r0 + r * RP + grp;
            on[r] = row < a.outer;
            at[r] = (size_t)(on[r] ? row : 0) * a.C;
            c[r] = 0.f;
        }
        if constexpr (K > 0) {
            // the rows to come are under way while these are worked on
            now = next;
            if (r0 + step < a.outer) fetch(r0 + step, next);
#pragma unroll
            for (int r = 0; r < R; ++r) rstd[r] = now.rstd[r];
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) rstd[r] = on[r] ? a.rstd[r0 + r * RP + grp] : 0.f;
        }
        auto &rx = now.x;
        auto &rd = now.d;
        auto &rh = now.h;
        const void *gamma = a.gamma;
        auto get = [&](const elem_t *x, int r, int v, const Part &p) { return on[r] && v < nv ? get_part<DT, SHORT>(x + at[r], p) : uint4{0, 0, 0, 0}; };
        rounds([&](int k, int v) {
            const Part p = part_of<V>(v, a.C, SHORT ? a.exact : 0);
            float g[V];
            if (v < nv) {
                load_gamma<DT, V, SHORT>(a, gamma, p, g);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) g[i] = 0.f;
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if constexpr (K == 0) {
                    rx[r][0] = get(H, r, v, p);
                    rd[r][0] = get(DY, r, v, p);
                }
                float x[V], d[V];
                unpack<DT>(rx[r][k], x);
                unpack<DT>(rd[r][k], d);
                if (K > 0 ? masked<G>(a, k, nv) : a.ragged) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const bool mine = on[r] && v < nv && own(p, i);
                        x[i] = mine ? x[i] : 0.f;
                        d[i] = mine ? d[i] : 0.f;
                    }
                }
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float t = d[i] * (x[i] * rstd[r]);
                    c[r] += t * g[i];
                    if constexpr (K > 0) {
                        ag[k][i] += t;
                    } else if (part && (!a.ragged || own(p, i))) {
                        float *q = part + p.at + i;
                        *q = (first ? 0.f : *q) + t;
                    }
                }
                if constexpr (K > 0) {
                    keep_packed(rx[r][k], ag[k]);
                    keep_packed(rd[r][k], ag[k]);
                }
            }
        });
        if (!DR && !DX) continue;
        // an output may lie over an input, part of which another lane's overlapping vector reads as well: all is read before anything is written
        if (K > 0 && a.over) __builtin_amdgcn_s_waitcnt(0);
        group_sum<G, R, T>(c, red, turn);
        rounds([&](int k, int v) {
            if (v >= nv) return;
            const Part p = part_of<V>(v, a.C, SHORT ? a.exact : 0);
            float g[V];
            load_gamma<DT, V, SHORT>(a, gamma, p, g);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (!on[r]) continue;
                if constexpr (K == 0) {
                    rx[r][0] = get(H, r, v, p);
                    rd[r][0] = get(DY, r, v, p);
                    if (DH) rh[r][0] = get(DH, r, v, p);
                }
                const float c1 = c[r] * a.inv_c;
                float x[V], d[V];
                unpack<DT>(rx[r][k], x);
                unpack<DT>(rd[r][k], d);
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = rstd[r] * (d[i] * g[i] - (x[i] * rstd[r]) * c1);
                if (DH) {
                    unpack<DT>(rh[r][k], d);
#pragma unroll
                    for (int i = 0; i < V; ++i) x[i] += d[i];
                }
                if (DR) put_part<DT, SHORT>(DR + at[r], pack<DT>(x), p);
                if (DX) {
                    if (a.drop.q16) drop_values<V>(a.drop, key, at[r] + p.at, a.fours, x);
                    put_part<DT, SHORT>(DX + at[r], pack<DT>(x), p);
                }
            }
        });
    }
    if (K == 0 || !part) return;
    // groups of one workgroup hold the same columns: added up in order of the groups
    if constexpr (RP > 1) {
        constexpr int W = G * V;
        __shared__ float cols[RP * W];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (k > 0) __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) cols[grp * W + lane * V + i] = ag[k][i];
            __syncthreads();
            for (int q = threadIdx.x; q < W; q += T) {
                const int v = k * G + q / V;
                if (v >= nv) continue;
                const Part p = part_of<V>(v, a.C, SHORT ? a.exact : 0);
                if (!own(p, q % V)) continue;
                float s = 0.f;
                for (int r = 0; r < RP; ++r) s += cols[r * W + q];
                part[p.at + q % V] = s;
            }
        }
    } else {
        rounds([&](int k, int v) {
            if (v >= nv) return;
            const Part p = part_of<V>(v, a.C, SHORT ? a.exact : 0);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (own(p, i)) part[p.at + i] = ag[k][i];
        });
    }
}

// ---- planes --------------------------------------------------------------------------------------------------------
// largest over the threads along the channels of N columns, along with column_sum's sums: what a wave has in front of it, what all have
// behind it (its barriers serve both)
template <int N, int TX> __device__ inline void column_max(uint32_t (&s)[N], uint32_t *red)
{
#pragma unroll
    for (int o = TX; o < 64; o <<= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = max(s[i], (uint32_t)__shfl_xor((int)s[i], o));
    if ((threadIdx.x & 63) < TX)
#pragma unroll
        for (int i = 0; i < N; ++i) red[((threadIdx.x >> 6) * TX + threadIdx.x % TX) * N + i] = s[i];
}
template <int N, int NW, int TX> __device__ inline void column_max_join(uint32_t (&s)[N], const uint32_t *red)
{
#pragma unroll 2
    for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = max(s[i], red[(w * TX + threadIdx.x % TX) * N + i]);
}

// WHOLE: planes of at least one vector whose last vectors overlap, the ordinary case
template <int DT, bool OUT8, int NW, int K, int TX, bool WHOLE>
__global__ __launch_bounds__(NW * 64) void rms_planes_fwd_kernel(RmsArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, TY = NW * (64 / TX), KR = K > 0 ? K : 1;
    __shared__ float red[2 * NW * TX * V];       // (two, taken in turn: no barrier stands behind the reading of one)
    __shared__ uint32_t redm[OUT8 ? 2 * NW * TX * V : 1];
    int turn = 0;
    const int ty = threadIdx.x / TX;
    const bool drops = !OUT8 && a.drop.q16;
    const uint64_t key = drops ? drop_key(a.drop) : 0;
    const TileRun run = tiles_of(a);
    auto rounds = [&](auto &&body) {
        if constexpr (K > 0) {
            const int t = again(ty);
#pragma unroll
            for (int k = 0; k < K; ++k) body(k, t + k * TY);
        } else {
            for (int c = ty; c < a.C; c += TY) body(0, c);
        }
    };
    for (long long tile = run.from; tile < run.to; tile += run.step) {
        const PlaneAt at = plane_at<V, TX>(a, tile);
        const elem_t *x = static_cast<const elem_t *>(a.x) + at.base;
        const elem_t *res = a.res ? static_cast<const elem_t *>(a.res) + at.base : nullptr;
        float h[KR][V];
        uint4 rx[KR], rr[KR];
        auto make = [&](int k, int c) {
            unpack<DT>(rx[k], h[k]);
            if (drops) drop_values<V>(a.drop, key, at.base + (size_t)c * a.inner + at.p.at, a.fours, h[k]);
            if (res) {
                float t[V];
                unpack<DT>(rr[k], t);
#pragma unroll
                for (int i = 0; i < V; ++i) h[k][i] += t[i];
            }
        };
        if constexpr (K > 0) {
            // four channels at a time: more would be under way than registers hold
#pragma unroll
            for (int k0 = 0; k0 < K; k0 += 4) {
                const int t = again(ty);
#pragma unroll
                for (int k = k0; k < min(K, k0 + 4); ++k) rx[k] = plane_get<DT, WHOLE>(a, x, at, t + k * TY);
                if (res)
#pragma unroll
                    for (int k = k0; k < min(K, k0 + 4); ++k) rr[k] = plane_get<DT, WHOLE>(a, res, at, t + k * TY);
#pragma unroll
                for (int k = k0; k < min(K, k0 + 4); ++k) make(k, t + k * TY);
                if constexpr (K > 4) __builtin_amdgcn_sched_barrier(0);
            }
        }
        auto value = [&](int k, int c) {
            if constexpr (K == 0) {
                rx[0] = plane_get<DT, WHOLE>(a, x, at, c);
                if (res) rr[0] = plane_get<DT, WHOLE>(a, res, at, c);
                make(0, c);
            }
        };
        float s[V];
        uint32_t m[V];
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = 0.f, m[i] = 0;
        rounds([&](int k, int c) {
            value(k, c);
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] += h[k][i] * h[k][i];      // (channels that do not exist are zeros)
            if (K > 0 && a.h && at.on && c < a.C) plane_put<DT, WHOLE>(a, static_cast<elem_t *>(a.h) + at.base, at, c, pack<DT>(h[k]));
            if constexpr (K > 0 || OUT8) {
                const float g = load_gamma1<DT>(a, min(c, a.C - 1));
#pragma unroll
                for (int i = 0; i < V; ++i) h[k][i] *= g;
            }
            if constexpr (OUT8) {
#pragma unroll
                for (int i = 0; i < V; ++i) m[i] = max(m[i], magnitude(h[k][i]));
            }
        });
        const int slot = turn * (NW * TX * V);
        turn ^= 1;
        if constexpr (OUT8) column_max<V, TX>(m, redm + slot);
        column_sum<V, NW, TX, true>(s, red + slot);
        float rstd[V], f[V];
        bool two[V], any = false;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            rstd[i] = rstd_of(s[i], a);
            f[i] = rstd[i];
            two[i] = false;
        }
        if constexpr (OUT8) {
            column_max_join<V, NW, TX>(m, redm + slot);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float most = __uint_as_float(max(magnitude(__uint_as_float(m[i]) * rstd[i]), __float_as_uint(kLeast8)));
                two[i] = factor8(rstd[i], a.top / most, f[i]);
                any |= two[i];
                if (ty == 0 && at.on && own(at.p, i)) a.scale[at.pos + i] = most / a.top;
            }
            if (K > 0 && any)
#pragma unroll
                for (int k = 0; k < KR; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) h[k][i] *= two[i] ? rstd[i] : 1.f;
        }
        if (!at.on) continue;
        rounds([&](int k, int c) {
            if (c >= a.C) return;
            if constexpr (K == 0) {
                value(k, c);
                if (a.h) plane_put<DT, WHOLE>(a, static_cast<elem_t *>(a.h) + at.base, at, c, pack<DT>(h[k]));
                const float g = load_gamma1<DT>(a, c);
#pragma unroll
                for (int i = 0; i < V; ++i) h[k][i] = h[k][i] * g * (OUT8 && two[i] ? rstd[i] : 1.f);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) h[k][i] *= f[i];
            if constexpr (OUT8) store8<V, !WHOLE>(static_cast<uint8_t *>(a.y) + at.base + (size_t)c * a.inner, at.p, h[k], a.int8);
            else plane_put<DT, WHOLE>(a, static_cast<elem_t *>(a.y) + at.base, at, c, pack<DT>(h[k]));
        });
        if (!OUT8 && ty == 0 && a.rstd) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (own(at.p, i)) a.rstd[at.pos + i] = rstd[i];
        }
    }
}

template <int DT, int NW, int K, int TX, bool WHOLE>
__global__ __launch_bounds__(NW * 64, 4) void rms_planes_bwd_kernel(RmsArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, TY = NW * (64 / TX), KR = K > 0 ? K : 1;
    __shared__ float red[2 * NW * TX * V];       // (two, taken in turn)
    int turn = 0;
    const int ty = threadIdx.x / TX, tx = threadIdx.x % TX;
    const elem_t *H = static_cast<const elem_t *>(a.x), *DY = static_cast<const elem_t *>(a.dy), *DH = static_cast<const elem_t *>(a.dh);
    elem_t *DR = static_cast<elem_t *>(a.y), *DX = static_cast<elem_t *>(a.h);
    const uint64_t key = a.drop.q16 ? drop_key(a.drop) : 0;
    float *part = a.part ? a.part + (size_t)blockIdx.x * a.C : nullptr;
    float ag[KR], gk[KR];
#pragma unroll
    for (int k = 0; k < KR; ++k) {
        ag[k] = 0.f;
        gk[k] = K <= 4 ? load_gamma1<DT>(a, min(ty + k * TY, a.C - 1)) : 0.f;
    }
    auto rounds = [&](auto &&body) {
        if constexpr (K > 0) {
            const int t = again(ty);
#pragma unroll
            for (int k = 0; k < K; ++k) body(k, t + k * TY);
        } else {
            for (int c = ty; c < a.C; c += TY) body(0, c);
        }
    };
    bool first = true;
    const TileRun run = tiles_of(a);
    if (K == 0 && part && run.from >= run.to)
        for (int c = threadIdx.x; c < a.C; c += NW * 64) part[c] = 0.f;
    for (long long tile = run.from; tile < run.to; tile += run.step, first = false) {
        const PlaneAt at = plane_at<V, TX>(a, tile);
        uint4 rx[KR], rd[KR], rh[KR];
        auto get = [&](int k, int c) {
            rx[k] = plane_get<DT, WHOLE>(a, H + at.base, at, c);
            rd[k] = plane_get<DT, WHOLE>(a, DY + at.base, at, c);
        };
        auto get_h = [&](int k, int c) { rh[k] = plane_get<DT, WHOLE>(a, DH + at.base, at, c); };
        if constexpr (K > 0) {
            rounds(get);
            if (DH && K <= 4) rounds(get_h);
        }
        float rstd[V], c1[V];
        if constexpr (WHOLE) {
            load_params<XCONV_F32, V>(a.rstd, Part{0, 0, V}, 0.f, rstd, at.pos);
#pragma unroll
            for (int i = 0; i < V; ++i) rstd[i] = at.on ? rstd[i] : 0.f;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) rstd[i] = at.on && i < at.p.hi ? a.rstd[at.pos + i] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) c1[i] = 0.f;
        rounds([&](int k, int c) {
            if constexpr (K == 0) get(0, c);
            float x[V], d[V], sg = 0.f;
            unpack<DT>(rx[k], x);
            unpack<DT>(rd[k], d);
            const float g = K > 0 && K <= 4 ? gk[k] : load_gamma1<DT>(a, min(c, a.C - 1));
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float t = d[i] * (x[i] * rstd[i]);
                c1[i] += t * g;
                sg += !a.ragged || i >= at.p.lo ? t : 0.f;
            }
            if constexpr (K > 0) {
                ag[k] += sg;
                keep_packed(rx[k], c1);
                keep_packed(rd[k], c1);
                if constexpr (K > 4) __builtin_amdgcn_sched_barrier(0);
            } else if (part) {
#pragma unroll
                for (int o = TX / 2; o >= 1; o >>= 1) sg += __shfl_xor(sg, o);
                if (tx == 0) part[c] = (first ? 0.f : part[c]) + sg;
            }
        });
        if (!DR && !DX) continue;
        column_sum<V, NW, TX, true>(c1, red + turn * (NW * TX * V));
        turn ^= 1;
        if (!at.on) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) c1[i] *= a.inv_c;
        rounds([&](int k, int c) {
            if (c >= a.C) return;
            if constexpr (K == 0) get(0, c);
            if (DH && (K == 0 || K > 4)) get_h(k, c);
            float x[V], d[V];
            unpack<DT>(rx[k], x);
            unpack<DT>(rd[k], d);
            const float g = K > 0 && K <= 4 ? gk[k] : load_gamma1<DT>(a, min(c, a.C - 1));
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = rstd[i] * (d[i] * g - (x[i] * rstd[i]) * c1[i]);
            if (DH) {
                unpack<DT>(rh[k], d);
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] += d[i];
            }
            if (DR) plane_put<DT, WHOLE>(a, DR + at.base, at, c, pack<DT>(x));
            if (DX) {
                if (a.drop.q16) drop_values<V>(a.drop, key, at.base + (size_t)c * a.inner + at.p.at, a.fours, x);
                plane_put<DT, WHOLE>(a, DX + at.base, at, c, pack<DT>(x));
            }
            __builtin_amdgcn_sched_barrier(0);      // (rounds beside each other would hold more values than there are registers)
        });
    }
    if (K == 0 || !part) return;
    rounds([&](int k, int c) {
        float sg = ag[k];
#pragma unroll
        for (int o = TX / 2; o >= 1; o >>= 1) sg += __shfl_xor(sg, o);
        if (tx == 0 && c < a.C) part[c] = sg;
    });
}

// dgamma[c] = sum over the n workgroups' partial sums, in order: a workgroup takes 32 columns, its 32 rows of threads share the sums
constexpr int kRmsJoinCols = 32, kRmsJoinThreads = 1024;
template <int WT> __global__ __launch_bounds__(kRmsJoinThreads) void rms_join_kernel(const float *part, int n, int C, void *dgamma)
{
    constexpr int RW = kRmsJoinThreads / kRmsJoinCols;
    __shared__ float red[kRmsJoinThreads / 64][kRmsJoinCols];
    const int col = threadIdx.x % kRmsJoinCols, w = threadIdx.x / kRmsJoinCols;
    const int c = blockIdx.x * kRmsJoinCols + col;
    float s = 0.f;
    if (c < C) {
#pragma unroll 16
        for (int b = w; b < n; b += RW) s += part[(size_t)b * C + c];
    }
    s += __shfl_xor(s, 32);
    if ((threadIdx.x & 63) < kRmsJoinCols) red[threadIdx.x >> 6][col] = s;
    __syncthreads();
    if (threadIdx.x >= kRmsJoinCols || c >= C) return;
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kRmsJoinThreads / 64; ++i) t += red[i][col];
    static_cast<typename NormElem<WT>::t *>(dgamma)[c] = norm_round<WT>(t);
}

// ---- launches ------------------------------------------------------------------------------------------------------
struct RmsShape {
    int G, K, R, T;   // rows: lanes a row, vectors a lane (0: read again), rows at once, threads a workgroup
    int NW;           // planes: waves a workgroup
    int V;
    int TX;           // planes: lanes along the positions
};

// The smallest group that holds a row with one vector a lane; past a wave several vectors a lane, then groups of several waves.  Forward,
// a wave to a row waits for no other, and a lane with five to eight vectors has enough under way: 8192 rows of 4096 fp16 26.4 us = 5.1
// TB/s with one wave of eight vectors, 26.6 with four of two; 5000 channels 32 us with two of five, 34 with four of three.  Backward the
// sums of dgamma take as many registers again, and waves count for more: 8192 rows of 4096 46 us with four of two (the rows to come under
// way), 62 with two of four, which leave registers for half the waves.
enum RmsPass { kRmsForward, kRmsForward8, kRmsBackward };
// the shapes that a pass has: up to eight vectors a lane forward; up to six in 8 bits, whose gamma takes registers beside h; two backward,
// where every vector takes 32 registers (sums of dgamma, three tensors, those of the rows to come)
constexpr bool rms_has(RmsPass pass, int G, int K)
{
    if (K < 2) return true;
    if (pass == kRmsBackward) return K == 2;
    if (G == 64) return K != 8 || pass == kRmsForward;
    if (pass == kRmsForward) return G < 1024 && (K == 5 || K == 6 || K == 8);
    return G < 1024 ? K >= 4 && K <= 6 : K == 4;
}

RmsShape rms_rows_shape(int dtype, int C, RmsPass pass)
{
    const bool backward = pass == kRmsBackward;
    const int V = dtype == XCONV_F32 ? 4 : 8, nv = ceil_div(C, V);
    auto threads = [&](int G) { return backward ? std::max(512, G) : G > 64 ? G : 256; };
    for (int G : {4, 8, 16, 32, 64})
        if (nv <= G) return {G, 1, 2, threads(G), 0, V, kNormTX};
    if (backward) {
        for (int G : {64, 128, 256, 512, 1024})
            if (nv <= 2 * G) return {G, 2, 1, threads(G), 0, V, kNormTX};
    } else {
        for (int K : {2, 3, 4})
            if (nv <= K * 64) return {64, K, 1, threads(64), 0, V, kNormTX};
        for (int G : {64, 128, 256, 512, 1024})
            for (int K : {4, 5, 6, 8})
                if (nv <= K * G && rms_has(pass, G, K)) return {G, K, 1, threads(G), 0, V, kNormTX};
    }
    return {1024, 0, 1, 1024, 0, V, kNormTX};
}
// A workgroup takes 8 lanes of positions (a line of 16-bit values, 128 bytes) with four channels a thread, which is what registers hold; past 256
// channels four lanes (half a line, whose other half a neighbour on the same die takes at the same time) rather than eight channels a
// thread: backward, 64 x 1024 x 28 x 28 fp16 179 us so and 232 with eight, 64 x 512 76 and 85; 256 x 256 157 and 148 with whole lines.
RmsShape rms_planes_shape(int dtype, int C)
{
    const int V = dtype == XCONV_F32 ? 4 : 8;
    for (int K : {1, 2, 4})
        if (C <= 32 * K) return {0, K, 1, 0, 4, V, 8};
    if (C <= 256) return {0, 4, 1, 0, 8, V, 8};
    for (int NW : {8, 16})
        if (C <= 64 * NW) return {0, 4, 1, 0, NW, V, 4};
    return {0, 0, 1, 0, 16, V, 8};
}

constexpr int kRmsBlocks = 512;            // most workgroups that leave partial sums, of 8 waves
constexpr long long kRmsGrid = 1 << 20;    // most workgroups of the forward pass

int rms_blocks(const xconv_norm_desc *d, const RmsShape &s, bool bwd)
{
    if (d->inner > 1) {
        const long long want = plane_tiles(d, s.V, s.TX);
        return (int)std::min<long long>(want > 8 ? (want + 7) / 8 * 8 : want, bwd ? 8 * kRmsBlocks / s.NW : kRmsGrid);     // (what the chip holds at once)
    }
    const int rows = s.T / s.G * s.R;
    return (int)std::min<long long>((d->outer + rows - 1) / rows, bwd ? kRmsBlocks : kRmsGrid);
}

template <int DT, int G, int K, int R> hipError_t go_rms_rows(const RmsArgs &a, RmsPass pass, int blocks, hipStream_t st)
{
    const dim3 grid((unsigned)blocks);
    constexpr int TF = rms_fwd_threads<G>, TB = G > 512 ? G : 512;
    if constexpr (rms_has(kRmsForward, G, K))
        if (pass == kRmsForward) hipLaunchKernelGGL((rms_rows_fwd_kernel<DT, false, G, K, R>), grid, dim3(TF), 0, st, a);
    if constexpr (rms_has(kRmsForward8, G, K))
        if (pass == kRmsForward8) hipLaunchKernelGGL((rms_rows_fwd_kernel<DT, true, G, K, R>), grid, dim3(TF), 0, st, a);
    if constexpr (rms_has(kRmsBackward, G, K))
        if (pass == kRmsBackward) hipLaunchKernelGGL((rms_rows_bwd_kernel<DT, G, K, R, TB>), grid, dim3(TB), 0, st, a);
    return hipGetLastError();
}
template <int DT> hipError_t go_rms_rows_shape(const RmsArgs &a, const RmsShape &s, RmsPass pass, int blocks, hipStream_t st)
{
    switch (s.G * 16 + s.K) {
    case 4 * 16 + 1: return go_rms_rows<DT, 4, 1, 2>(a, pass, blocks, st);
    case 8 * 16 + 1: return go_rms_rows<DT, 8, 1, 2>(a, pass, blocks, st);
    case 16 * 16 + 1: return go_rms_rows<DT, 16, 1, 2>(a, pass, blocks, st);
    case 32 * 16 + 1: return go_rms_rows<DT, 32, 1, 2>(a, pass, blocks, st);
    case 64 * 16 + 1: return go_rms_rows<DT, 64, 1, 2>(a, pass, blocks, st);
    case 64 * 16 + 2: return go_rms_rows<DT, 64, 2, 1>(a, pass, blocks, st);
    case 64 * 16 + 3: return go_rms_rows<DT, 64, 3, 1>(a, pass, blocks, st);
    case 64 * 16 + 4: return go_rms_rows<DT, 64, 4, 1>(a, pass, blocks, st);
    case 64 * 16 + 5: return go_rms_rows<DT, 64, 5, 1>(a, pass, blocks, st);
    case 64 * 16 + 6: return go_rms_rows<DT, 64, 6, 1>(a, pass, blocks, st);
    case 64 * 16 + 8: return go_rms_rows<DT, 64, 8, 1>(a, pass, blocks, st);
    case 128 * 16 + 2: return go_rms_rows<DT, 128, 2, 1>(a, pass, blocks, st);
    case 128 * 16 + 4: return go_rms_rows<DT, 128, 4, 1>(a, pass, blocks, st);
    case 128 * 16 + 5: return go_rms_rows<DT, 128, 5, 1>(a, pass, blocks, st);
    case 128 * 16 + 6: return go_rms_rows<DT, 128, 6, 1>(a, pass, blocks, st);
    case 128 * 16 + 8: return go_rms_rows<DT, 128, 8, 1>(a, pass, blocks, st);
    case 256 * 16 + 2: return go_rms_rows<DT, 256, 2, 1>(a, pass, blocks, st);
    case 256 * 16 + 4: return go_rms_rows<DT, 256, 4, 1>(a, pass, blocks, st);
    case 256 * 16 + 5: return go_rms_rows<DT, 256, 5, 1>(a, pass, blocks, st);
    case 256 * 16 + 6: return go_rms_rows<DT, 256, 6, 1>(a, pass, blocks, st);
    case 256 * 16 + 8: return go_rms_rows<DT, 256, 8, 1>(a, pass, blocks, st);
    case 512 * 16 + 2: return go_rms_rows<DT, 512, 2, 1>(a, pass, blocks, st);
    case 512 * 16 + 4: return go_rms_rows<DT, 512, 4, 1>(a, pass, blocks, st);
    case 512 * 16 + 5: return go_rms_rows<DT, 512, 5, 1>(a, pass, blocks, st);
    case 512 * 16 + 6: return go_rms_rows<DT, 512, 6, 1>(a, pass, blocks, st);
    case 512 * 16 + 8: return go_rms_rows<DT, 512, 8, 1>(a, pass, blocks, st);
    case 1024 * 16 + 2: return go_rms_rows<DT, 1024, 2, 1>(a, pass, blocks, st);
    case 1024 * 16 + 4: return go_rms_rows<DT, 1024, 4, 1>(a, pass, blocks, st);
    default: return go_rms_rows<DT, 1024, 0, 1>(a, pass, blocks, st);
    }
}
template <int DT, int NW, int K, int TX, bool WHOLE> hipError_t go_rms_planes(const RmsArgs &a, RmsPass pass, int blocks, hipStream_t st)
{
    const dim3 grid((unsigned)blocks), block(NW * 64);
    if (pass == kRmsForward) hipLaunchKernelGGL((rms_planes_fwd_kernel<DT, false, NW, K, TX, WHOLE>), grid, block, 0, st, a);
    else if (pass == kRmsForward8) hipLaunchKernelGGL((rms_planes_fwd_kernel<DT, true, NW, K, TX, WHOLE>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((rms_planes_bwd_kernel<DT, NW, K, TX, WHOLE>), grid, block, 0, st, a);
    return hipGetLastError();
}
template <int DT, bool WHOLE> hipError_t go_rms_planes_shape(const RmsArgs &a, const RmsShape &s, RmsPass pass, int blocks, hipStream_t st)
{
    switch ((s.NW * 8 + s.K) * 8 + s.TX % 8) {
    case (4 * 8 + 1) * 8 + 0: return go_rms_planes<DT, 4, 1, 8, WHOLE>(a, pass, blocks, st);
    case (4 * 8 + 2) * 8 + 0: return go_rms_planes<DT, 4, 2, 8, WHOLE>(a, pass, blocks, st);
    case (4 * 8 + 4) * 8 + 0: return go_rms_planes<DT, 4, 4, 8, WHOLE>(a, pass, blocks, st);
    case (8 * 8 + 4) * 8 + 0: return go_rms_planes<DT, 8, 4, 8, WHOLE>(a, pass, blocks, st);
    case (8 * 8 + 4) * 8 + 4: return go_rms_planes<DT, 8, 4, 4, WHOLE>(a, pass, blocks, st);
    case (16 * 8 + 4) * 8 + 4: return go_rms_planes<DT, 16, 4, 4, WHOLE>(a, pass, blocks, st);
    default: return go_rms_planes<DT, 16, 0, 8, WHOLE>(a, pass, blocks, st);
    }
}

template <int DT> hipError_t launch_rms_dt(const xconv_norm_desc *d, RmsArgs a, RmsPass pass, void *dgamma, hipStream_t st)
{
    const bool planes = d->inner > 1, bwd = pass == kRmsBackward;
    constexpr int V = NormElem<DT>::V;
    // outputs over inputs: the overlapping part of a plane may be another workgroup's, that of a row read again another lane's
    const size_t bytes = (size_t)d->outer * d->C * d->inner * (DT == XCONV_F32 ? 4 : 2);
    bool over = false;
    for (const void *out : {pass == kRmsForward8 ? nullptr : a.y, a.h})
        for (const void *in : {a.x, a.res, a.dy, a.dh}) over = over || overlap(out, in, bytes);
    const RmsShape s = planes ? rms_planes_shape(DT, d->C) : rms_rows_shape(DT, d->C, pass);
    a.over = over;
    a.ragged = (planes ? d->inner : (int64_t)d->C) % V != 0;
    a.exact = planes ? over || d->inner < V : d->C < V || (s.K == 0 && over);
    a.outer = d->outer;
    a.C = d->C;
    a.inner = (int)d->inner;
    a.eps = d->eps;
    a.count = (float)d->C;
    a.inv_c = 1.0f / a.count;
    a.nvi = ceil_div((int)d->inner, s.V);
    a.tiles = plane_tiles(d, s.V, s.TX);
    a.w32 = d->w_dtype == XCONV_F32;
    a.fours = (planes ? d->inner : (int64_t)d->C) % 4 == 0;
    const int blocks = rms_blocks(d, s, bwd);
    hipError_t e = hipSuccess;
    if (d->outer > 0) {
        if (!planes) e = go_rms_rows_shape<DT>(a, s, pass, blocks, st);
        else if (a.exact) e = go_rms_planes_shape<DT, false>(a, s, pass, blocks, st);
        else e = go_rms_planes_shape<DT, true>(a, s, pass, blocks, st);
    }
    if (e != hipSuccess || !dgamma) return e;
    const dim3 grid((unsigned)ceil_div(d->C, kRmsJoinCols));
    if (a.w32) hipLaunchKernelGGL(rms_join_kernel<XCONV_F32>, grid, dim3(kRmsJoinThreads), 0, st, a.part, blocks, d->C, dgamma);
    else hipLaunchKernelGGL(rms_join_kernel<DT>, grid, dim3(kRmsJoinThreads), 0, st, a.part, blocks, d->C, dgamma);
    return hipGetLastError();
}

hipError_t launch_rms(const xconv_norm_desc *d, const RmsArgs &a, RmsPass pass, void *dgamma, hipStream_t st)
{
    if (d->dtype == XCONV_F32) return launch_rms_dt<XCONV_F32>(d, a, pass, dgamma, st);
    if (d->dtype == XCONV_BF16) return launch_rms_dt<XCONV_BF16>(d, a, pass, dgamma, st);
    return launch_rms_dt<XCONV_F16>(d, a, pass, dgamma, st);
}

}  // namespace

size_t rms_ws_bytes(const xconv_norm_desc *d)
{
    const RmsShape s = d->inner > 1 ? rms_planes_shape(d->dtype, d->C) : rms_rows_shape(d->dtype, d->C, kRmsBackward);
    return (size_t)rms_blocks(d, s, true) * d->C * sizeof(float);
}

hipError_t launch_rms_fwd(const xconv_norm_desc *d, const void *X, const void *residual, const void *gamma, void *Y, void *H, float *rstd, const xconv_drop *drop,
                          hipStream_t st)
{
    RmsArgs a{};
    a.x = X; a.res = residual; a.gamma = gamma; a.y = Y; a.h = H; a.rstd = rstd;
    a.drop = drop_args(drop);
    return launch_rms(d, a, kRmsForward, nullptr, st);
}

hipError_t launch_rms_fwd8(const xconv_norm_desc *d, bool int8, const void *X, const void *residual, const void *gamma, void *Q, float *scale, void *H, hipStream_t st)
{
    RmsArgs a{};
    a.x = X; a.res = residual; a.gamma = gamma; a.y = Q; a.h = H; a.scale = scale;
    a.int8 = int8;
    a.top = int8 ? 127.f : 448.f;
    a.drop = drop_args(nullptr);
    return launch_rms(d, a, kRmsForward8, nullptr, st);
}

hipError_t launch_rms_bwd(const xconv_norm_desc *d, const void *dY, const void *H, const float *rstd, const void *gamma, const void *dH, void *dX, void *dR,
                          void *dgamma, float *part, const xconv_drop *drop, hipStream_t st)
{
    RmsArgs a{};
    a.x = H; a.dy = dY; a.dh = dH; a.gamma = gamma; a.y = dR; a.h = dX;
    a.rstd = const_cast<float *>(rstd);
    a.part = dgamma ? part : nullptr;
    a.drop = drop_args(drop);
    return launch_rms(d, a, kRmsBackward, dgamma, st);
}

}  // namespace xc
