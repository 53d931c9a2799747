// Layer normalisation over the channels of every position, forward and backward.
//     forward   mean = sum_c x / C, var = sum_c (x - mean)^2 / C, rstd = 1 / sqrt(var + eps), y = (x - mean) rstd gamma + beta
//     backward  g = dy gamma, xh = (x - mean) rstd, dx = rstd (g - sum_c g / C - xh sum_c (g xh) / C),
//               dgamma = sum over positions of dy xh, dbeta = sum over positions of dy
// X is [outer, C, inner]: inner == 1 are rows (channels-last activations), inner > 1 planes.  Sums are fp32; the variance is
// summed from the centred values (a mean far from zero costs no digits), every output is rounded once.
// Bound by HBM: every tensor is read once, its values stay in registers between the statistics and the output.
//
// Rows: a group of G lanes (part of a wave, a wave, or a workgroup) holds R rows, K 16-byte vectors a row and lane, and sums
// across lanes.  Planes: 8 lanes lie along the positions (one 128-byte line of a plane), the other threads along the channels,
// K channels each; sums across threads go through LDS.  Longer rows and more channels than the registers hold are read
// again from the cache (K == 0).  Rows and planes of any length are read as vectors at the alignment of an element, which the
// memory system takes; the last vector of one whose length is no multiple of V starts earlier and overlaps the one before it.
//
// Backward: a fixed number of workgroups walks the positions and adds up dgamma and dbeta in registers, in fixed order; their
// partial sums are added up in order by a second launch, so that results do not depend on timing.
//
// Measured (three sets of tensors in turn): forward, 200704 rows of 128 bf16, 20.5 us = 5.0 TB/s, the rate of a large copy (5.2);
// 2049 rows of 5001 fp16, 13.6 us = 3.0 TB/s (a workgroup a row, two sums through LDS; unmasked whole rows would be the same);
// backward, 131072 rows of 64 fp32, 18.5 us = 5.4 TB/s and 3.8 us for the join; 256 x 256 x 28 x 28 fp16 planes, 76 us = 4.0 TB/s
// and 5 us (the plane of 1568 bytes is no whole lines: lines at the tiles' edges are fetched by two workgroups).
// Further from a copy's rate: backward over few long rows, where the partial sums of up to 1024 workgroups are 8 C bytes each, written and
// read again (4096 x 4096 bf16 54 us, 34 MB of them beside 100 MB of tensors; 2048 x 8192 97 us, 67 MB); and the shapes whose backward
// pass keeps registers in scratch: planes of 513 to 1024 channels (33 of a thread's in fp32, 96 to 98 in 16 bits: 64 x 1024 x 28 x 28 fp16
// 202 us = 1.5 TB/s), 16-bit rows of 16385 to 24576 channels (63), and four of them in 16-bit planes of 65 to 512 channels.
#include <algorithm>

#include "common.h"
#include "launch.h"

namespace xc {

namespace {

template <int DT> struct NormElem { typedef uint16_t t; static constexpr int V = 8; };
template <> struct NormElem<XCONV_F32> { typedef float t; static constexpr int V = 4; };

template <int DT> __device__ inline float norm_val(typename NormElem<DT>::t v)
{
    if constexpr (DT == XCONV_F32) return v;
    else return st16_to_f32<DT>(v);
}
template <int DT> __device__ inline typename NormElem<DT>::t norm_round(float v)
{
    if constexpr (DT == XCONV_F32) return v;
    else return f32_to_st16<DT>(v);
}

// 16 bytes at the alignment of an element
template <int DT> struct __attribute__((packed, aligned(DT == XCONV_F32 ? 4 : 2))) Loose { uint32_t w[4]; };
template <int DT> __device__ inline uint4 load_loose(const typename NormElem<DT>::t *p) 
{
    const Loose<DT> v = *reinterpret_cast<const Loose<DT> *>(p);
    return uint4{v.w[0], v.w[1], v.w[2], v.w[3]};
}
template <int DT> __device__ inline void store_loose(typename NormElem<DT>::t *p, const uint4 &v) 
{
    *reinterpret_cast<Loose<DT> *>(p) = Loose<DT>{{v.x, v.y, v.z, v.w}};
}

struct NormArgs {
    const void *x, *dy, *gamma, *beta;
    void *y;              // y or dx
    float *mean, *rstd;   // written (forward, may be null) or read (backward)
    float *part;          // backward: [workgroups][2][C] partial sums of dgamma and dbeta, null when neither is wanted
    long long outer;
    int C, inner;
    float eps, inv_c, count;   // count = C, inv_c = 1 / C
    int nvi;              // vectors a plane
    long long tiles;      // tiles of kNormTX vectors of positions (planes)
    int ragged;           // rows (planes) are no whole number of vectors: values that are not a vector's own are masked
    int exact;            // last vectors do not overlap (shorter than a vector; outputs over inputs that are read again)
};

// Vector v of a run of n values: values lo .. hi - 1 of the V from `at` on are the vector's own.  Those below lo belong to the
// vector before it as well: they are computed twice, with the same result, and count once in every sum.
struct Part {
    int at, lo, hi;
};
template <int V> __device__ inline Part part_of(int v, int n, int exact)
{
    if (exact) return {v * V, 0, min(V, n - v * V)};
    const int at = min(v * V, n - V);
    return {at, v * V - at, V};
}
__device__ inline bool own(const Part &p, int i) { return i >= p.lo && i < p.hi; }

// the first n < V values, in runs of 4, 2 and 1
template <int DT> __device__ inline uint4 load_short(const typename NormElem<DT>::t *p, int n)
{
    uint4 v{0, 0, 0, 0};
    if constexpr (DT == XCONV_F32) {
        v.x = n > 0 ? __float_as_uint(p[0]) : 0u;
        v.y = n > 1 ? __float_as_uint(p[1]) : 0u;
        v.z = n > 2 ? __float_as_uint(p[2]) : 0u;
    } else {
        auto pair = [&](int i) { return (n > i ? (uint32_t)p[i] : 0u) | (n > i + 1 ? (uint32_t)p[i + 1] << 16 : 0u); };
        v = uint4{pair(0), pair(2), pair(4), pair(6)};
    }
    return v;
}
template <int DT> __device__ inline void store_short(typename NormElem<DT>::t *p, const uint4 v, int n)
{
    constexpr int V = NormElem<DT>::V;
    struct Pack { typename NormElem<DT>::t e[V]; };
    const Pack k = __builtin_bit_cast(Pack, v);
#pragma unroll
    for (int i = 0; i < V - 1; ++i)
        if (i < n) p[i] = k.e[i];
}
template <int DT> __device__ inline uint4 load_part(const typename NormElem<DT>::t *run, const Part &p)
{
    return p.hi == NormElem<DT>::V ? load_loose<DT>(run + p.at) : load_short<DT>(run + p.at, p.hi);
}
template <int DT> __device__ inline void store_part(typename NormElem<DT>::t *run, const uint4 &v, const Part &p)
{
    if (p.hi == NormElem<DT>::V) store_loose<DT>(run + p.at, v);
    else store_short<DT>(run + p.at, v, p.hi);
}
template <int DT> __device__ inline void unpack(const uint4 &v, float (&x)[NormElem<DT>::V])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DT == XCONV_F32) {
            x[i] = __uint_as_float(w[i]);
        } else {
            x[2 * i] = st16_to_f32<DT>((uint16_t)(w[i] & 0xffffu));
            x[2 * i + 1] = st16_to_f32<DT>((uint16_t)(w[i] >> 16));
        }
    }
}
template <int DT> __device__ inline uint4 pack(const float (&x)[NormElem<DT>::V])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DT == XCONV_F32) w[i] = __float_as_uint(x[i]);
        else if constexpr (DT == XCONV_BF16) w[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
        else w[i] = (uint32_t)f32_to_st16<DT>(x[2 * i]) | (uint32_t)f32_to_st16<DT>(x[2 * i + 1]) << 16;
    }
    return uint4{w[0], w[1], w[2], w[3]};
}
// Keeps 16 bytes as they are: what follows unpacks them again instead of holding the unpacked values in twice the registers.
// The sums that were just made of them are operands too, so that those come first.
template <int N> __device__ inline void keep_packed(uint4 &v, float (&sums)[N])
{
    asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w));
#pragma unroll
    for (int i = 0; i < N; i += 4) asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w), "+v"(sums[i]), "+v"(sums[i + 1]), "+v"(sums[i + 2]), "+v"(sums[i + 3]));
}

// V parameters of the type WT from p.at on, those that exist
template <int WT, int V> __device__ inline void load_params(const void *q, const Part &p, float none, float (&out)[V], long long from = 0)
{
    typedef typename NormElem<WT>::t elem_t;
    const elem_t *e = static_cast<const elem_t *>(q) + from + p.at;
    constexpr int VW = NormElem<WT>::V;
    if (!q) {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = none;
    } else if (p.hi == V && V >= VW) {
#pragma unroll
        for (int j = 0; j < V; j += VW) {
            float t[VW];
            unpack<WT>(load_loose<WT>(e + j), t);
#pragma unroll
            for (int i = 0; i < VW; ++i) out[j + i] = t[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = i < p.hi ? norm_val<WT>(e[i]) : none;
    }
}
template <int WT> __device__ inline float load_param(const void *p, int c, float none)
{
    return p ? norm_val<WT>(static_cast<const typename NormElem<WT>::t *>(p)[c]) : none;
}

// s / count to the last bit but rare ones, at a quarter of a division's instructions; 1 / sqrt(v) to one unit in the last place
__device__ inline float mean_of(float s, const NormArgs &a)
{
    const float q = s * a.inv_c;
    return fabsf(q) < 1e30f ? fmaf(fmaf(-q, a.count, s), a.inv_c, q) : q;
}
__device__ inline float rstd_of(float squares, const NormArgs &a) { return rsqrtf(squares * a.inv_c + a.eps); }

// sums of R values over a group of G lanes of a wave, or over the workgroup's G threads through `red` (two slots of R * G / 64
// floats, taken in turn so that one barrier a sum is enough)
template <int G, int R> __device__ inline void group_sum(float (&s)[R], float *red, int &turn)
{
#pragma unroll
    for (int o = (G < 64 ? G : 64) / 2; o >= 1; o >>= 1)
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] += __shfl_xor(s[r], o);
    if constexpr (G > 64) {
        constexpr int W = G / 64;
        float *slot = red + turn * W * R;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int r = 0; r < R; ++r) slot[(threadIdx.x >> 6) * R + r] = s[r];
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r) s[r] += slot[i * R + r];
    }
}

// ---- rows ----------------------------------------------------------------------------------------------------------
// whether the wave's round k of vectors needs masks: rows that are no whole vectors, in the wave that has the last one
template <int G> __device__ inline bool masked(const NormArgs &a, int k, int nv)
{
    if constexpr (G <= 64) return a.ragged;
    else return a.ragged && __builtin_amdgcn_readfirstlane((int)(threadIdx.x % G) | 63) + k * G >= nv - 1;
}

// G lanes a row, K vectors a lane (lane l holds vectors l, l + G, ...), R rows at once; K == 0: a row is read once a pass.
template <int G> constexpr int row_threads = G > 256 ? G : 256;

template <int DT, int WT, int G, int K, int R>
__global__ __launch_bounds__(row_threads<G>) void norm_rows_fwd_kernel(NormArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, RP = row_threads<G> / G, KR = K > 0 ? K : 1;
    __shared__ float red[G > 64 ? 2 * R * (G / 64) : 1];
    int turn = 0;
    const int lane = threadIdx.x % G, grp = threadIdx.x / G;
    const int nv = (a.C + V - 1) / V;
    const elem_t *X = static_cast<const elem_t *>(a.x);
    elem_t *Y = static_cast<elem_t *>(a.y);
    // the rounds of vectors: k of the registers, or all that there are
    auto rounds = [&](auto &&body) {
        if constexpr (K > 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) body(k, lane + k * G);
        } else {
            for (int v = lane; v < nv; v += G) body(0, v);
        }
    };
    for (long long r0 = (long long)blockIdx.x * (RP * R); r0 < a.outer; r0 += (long long)gridDim.x * (RP * R)) {   // (the same count for all threads)
        uint4 raw[R][KR];
        long long row[R];
        bool on[R];
        const elem_t *x[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            row[r] = r0 + r * RP + grp;
            on[r] = row[r] < a.outer;
            x[r] = X + (size_t)(on[r] ? row[r] : 0) * a.C;
        }
        if constexpr (K > 0)
            rounds([&](int k, int v) {
                const Part p = part_of<V>(v, a.C, a.exact);
#pragma unroll
                for (int r = 0; r < R; ++r) raw[r][k] = v < nv ? load_part<DT>(x[r], p) : uint4{0, 0, 0, 0};
            });
        auto value = [&](int r, int k, const Part &p) -> uint4 {
            if constexpr (K > 0) return raw[r][k];
            else return load_part<DT>(x[r], p);
        };
        float s[R], mean[R], rstd[R];
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = 0.f;
        rounds([&](int k, int v) {
            const Part p = part_of<V>(v, a.C, a.exact);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float t[V];
                unpack<DT>(value(r, k, p), t);
                if (K > 0 ? !masked<G>(a, k, nv) : !a.ragged) {
#pragma unroll
                    for (int i = 0; i < V; ++i) s[r] += t[i];       // (zeros past the last vector)
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) s[r] += v < nv && own(p, i) ? t[i] : 0.f;
                }
            }
        });
        group_sum<G>(s, red, turn);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean[r] = mean_of(s[r], a);
            s[r] = 0.f;
        }
        rounds([&](int k, int v) {
            const Part p = part_of<V>(v, a.C, a.exact);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float t[V];
                unpack<DT>(value(r, k, p), t);
                float q = 0.f;
                if (K > 0 ? !masked<G>(a, k, nv) : !a.ragged) {
#pragma unroll
                    for (int i = 0; i < V; ++i) q += (t[i] - mean[r]) * (t[i] - mean[r]);
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float d = own(p, i) ? t[i] - mean[r] : 0.f;
                        q += d * d;
                    }
                }
                s[r] += v < nv ? q : 0.f;
            }
        });
        group_sum<G>(s, red, turn);
#pragma unroll
        for (int r = 0; r < R; ++r) rstd[r] = rstd_of(s[r], a);
        rounds([&](int k, int v) {
            if (v >= nv) return;
            const Part p = part_of<V>(v, a.C, a.exact);
            float g[V], b[V];
            load_params<WT, V>(a.gamma, p, 1.f, g);
            load_params<WT, V>(a.beta, p, 0.f, b);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (!on[r]) continue;
                float t[V];
                unpack<DT>(value(r, k, p), t);
#pragma unroll
                for (int i = 0; i < V; ++i) t[i] = (t[i] - mean[r]) * rstd[r] * g[i] + b[i];
                store_part<DT>(Y + (size_t)row[r] * a.C, pack<DT>(t), p);
            }
        });
        if (lane == 0) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (on[r]) {
                    if (a.mean) a.mean[row[r]] = mean[r];
                    if (a.rstd) a.rstd[row[r]] = rstd[r];
                }
        }
    }
}

// A workgroup's groups walk the rows; every lane adds up dgamma and dbeta of its own columns.  K == 0: one row a workgroup at
// a time, dgamma and dbeta in the workgroup's own slots of `part`.
template <int DT, int WT, int G, int K, int R>
__global__ __launch_bounds__(row_threads<G>) void norm_rows_bwd_kernel(NormArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, T = row_threads<G>, RP = T / G, KR = K > 0 ? K : 1;
    __shared__ float red[G > 64 ? 4 * R * (G / 64) : 1];
    int turn = 0;
    const int lane = threadIdx.x % G, grp = threadIdx.x / G;
    const elem_t *X = static_cast<const elem_t *>(a.x), *DY = static_cast<const elem_t *>(a.dy);
    elem_t *DX = static_cast<elem_t *>(a.y);
    const int nv = (a.C + V - 1) / V;
    float *part = a.part ? a.part + (size_t)blockIdx.x * 2 * a.C : nullptr;
    auto rounds = [&](auto &&body) {
        if constexpr (K > 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) body(k, lane + k * G);
        } else {
            for (int v = lane; v < nv; v += G) body(0, v);
        }
    };
    float ag[KR][V], ab[KR][V];
#pragma unroll
    for (int k = 0; k < KR; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) ag[k][i] = ab[k][i] = 0.f;
    bool first = true;
    for (long long r0 = (long long)blockIdx.x * (RP * R); r0 < a.outer; r0 += (long long)gridDim.x * (RP * R), first = false) {   // (the same count for all threads)
        uint4 rx[R][KR], rd[R][KR];
        float mean[R], rstd[R], c[2 * R];
        size_t at[R];
        bool on[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long row = r0 + r * RP + grp;
            on[r] = row < a.outer;
            at[r] = (size_t)(on[r] ? row : 0) * a.C;
            mean[r] = on[r] ? a.mean[row] : 0.f;
            rstd[r] = on[r] ? a.rstd[row] : 0.f;
            c[2 * r] = c[2 * r + 1] = 0.f;
        }
        auto get = [&](int r, int k, int v, const Part &p) {
            const bool has = on[r] && v < nv;
            rx[r][k] = has ? load_part<DT>(X + at[r], p) : uint4{0, 0, 0, 0};
            rd[r][k] = has ? load_part<DT>(DY + at[r], p) : uint4{0, 0, 0, 0};
        };
        if constexpr (K > 0)
            rounds([&](int k, int v) {
                const Part p = part_of<V>(v, a.C, a.exact);
#pragma unroll
                for (int r = 0; r < R; ++r) get(r, k, v, p);
            });
        rounds([&](int k, int v) {
            const Part p = part_of<V>(v, a.C, a.exact);
            float g[V];
            if (v < nv) {
                load_params<WT, V>(a.gamma, p, 1.f, g);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) g[i] = 0.f;
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if constexpr (K == 0) get(r, k, v, p);
                float x[V], d[V];
                unpack<DT>(rx[r][k], x);
                unpack<DT>(rd[r][k], d);
                // (rows and vectors that do not exist are zeros with a mean of zero)
                const float mu = v < nv ? mean[r] : 0.f;
                if (K > 0 ? masked<G>(a, k, nv) : a.ragged) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const bool mine = on[r] && v < nv && own(p, i);
                        x[i] = mine ? x[i] : mu;
                        d[i] = mine ? d[i] : 0.f;
                    }
                }
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float t = d[i] * ((x[i] - mu) * rstd[r]);
                    c[2 * r] += d[i] * g[i];
                    c[2 * r + 1] += t * g[i];
                    if constexpr (K > 0) {
                        ag[k][i] += t;
                        ab[k][i] += d[i];
                    } else if (part && (!a.ragged || own(p, i))) {
                        float *pg = part + p.at + i, *pb = pg + a.C;
                        *pg = (first ? 0.f : *pg) + t;
                        *pb = (first ? 0.f : *pb) + d[i];
                    }
                }
                if constexpr (K > 1) {
                    keep_packed(rx[r][k], ag[k]);
                    keep_packed(rd[r][k], ab[k]);
                }
            }
        });
        if (!DX) continue;
        group_sum<G>(c, red, turn);
        rounds([&](int k, int v) {
            if (v >= nv) return;
            const Part p = part_of<V>(v, a.C, a.exact);
            float g[V];
            load_params<WT, V>(a.gamma, p, 1.f, g);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (!on[r]) continue;
                if constexpr (K == 0) get(r, k, v, p);
                const float c1 = c[2 * r] * a.inv_c * rstd[r], c2 = c[2 * r + 1] * a.inv_c * rstd[r] * rstd[r];
                float x[V], d[V];
                unpack<DT>(rx[r][k], x);
                unpack<DT>(rd[r][k], d);
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = (d[i] * (g[i] * rstd[r]) - c1) - (x[i] - mean[r]) * c2;
                store_part<DT>(DX + at[r], pack<DT>(x), p);
            }
        });
    }
    if (K == 0 || !part) return;
    // groups of one workgroup hold the same columns: added up in order of the groups
    constexpr int W = G * KR * V;
    if constexpr (RP > 1) {
        extern __shared__ float cols[];     // [RP][2][W]
        rounds([&](int k, int v) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                cols[(grp * 2) * W + v * V + i] = ag[k][i];
                cols[(grp * 2 + 1) * W + v * V + i] = ab[k][i];
            }
        });
        __syncthreads();
        for (int q = threadIdx.x; q < 2 * W; q += T) {
            const int slot = q % W;
            if (slot / V >= nv) continue;
            const Part p = part_of<V>(slot / V, a.C, a.exact);
            if (!own(p, slot % V)) continue;
            float s = 0.f;
            for (int r = 0; r < RP; ++r) s += cols[r * 2 * W + q];
            part[(size_t)(q / W) * a.C + p.at + slot % V] = s;
        }
    } else {
        rounds([&](int k, int v) {
            if (v >= nv) return;
            const Part p = part_of<V>(v, a.C, a.exact);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (own(p, i)) {
                    part[p.at + i] = ag[k][i];
                    part[(size_t)a.C + p.at + i] = ab[k][i];
                }
        });
    }
}

// ---- planes --------------------------------------------------------------------------------------------------------
constexpr int kNormTX = 8;               // lanes along the positions
constexpr int kNormTYW = 64 / kNormTX;   // channels of a wave

// sums over the threads along the channels of N columns of V positions each; `red` [NW][kNormTX][N * V]
template <int N, int NW> __device__ inline void column_sum(float (&s)[N], float *red)
{
#pragma unroll
    for (int o = kNormTX; o < 64; o <<= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += __shfl_xor(s[i], o);
    const int tx = threadIdx.x % kNormTX;
    __syncthreads();                     // whoever still reads the last sum
    if ((threadIdx.x & 63) < kNormTX)
#pragma unroll
        for (int i = 0; i < N; ++i) red[((threadIdx.x >> 6) * kNormTX + tx) * N + i] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = 0.f;
#pragma unroll 2
    for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += red[(w * kNormTX + tx) * N + i];
}

// where the thread's vector of positions lies: first value of channel 0 of the image, its first position, the vector's part
struct PlaneAt {
    size_t base;
    long long pos;
    Part p;
    bool on;
};
template <int V> __device__ inline PlaneAt plane_at(const NormArgs &a, long long tile)
{
    const long long q = tile * kNormTX + threadIdx.x % kNormTX;
    const long long img = a.tiles * kNormTX < (1LL << 31) ? (long long)((uint32_t)q / (uint32_t)a.nvi) : q / a.nvi;
    if (img >= a.outer) return {0, 0, {0, 0, V}, false};
    const Part p = part_of<V>((int)(q - img * a.nvi), a.inner, a.exact);
    return {(size_t)img * a.C * a.inner, img * a.inner + p.at, p, true};
}
// channel c of the vector; WHOLE: the planes are whole or overlapping vectors, and every lane loads (where there is nothing: zeros, or
// with ANY the values of another channel or position)
template <int DT, bool WHOLE, bool ANY = false> __device__ inline uint4 plane_get(const NormArgs &a, const typename NormElem<DT>::t *x, const PlaneAt &at, int c)
{
    const bool on = at.on && c < a.C;
    if constexpr (WHOLE) {
        const uint4 v = load_loose<DT>(x + (size_t)min(c, a.C - 1) * a.inner + at.p.at);
        if constexpr (ANY) return v;
        return uint4{on ? v.x : 0u, on ? v.y : 0u, on ? v.z : 0u, on ? v.w : 0u};
    } else {
        return on ? load_part<DT>(x + (size_t)c * a.inner, at.p) : uint4{0, 0, 0, 0};
    }
}
template <int DT, bool WHOLE> __device__ inline void plane_put(const NormArgs &a, typename NormElem<DT>::t *y, const PlaneAt &at, int c, const uint4 &v)
{
    if constexpr (WHOLE) store_loose<DT>(y + (size_t)c * a.inner + at.p.at, v);
    else store_part<DT>(y + (size_t)c * a.inner, v, at.p);
}
// The tiles of a workgroup.  Planes are rarely whole lines, so neighbouring tiles share lines of memory: each of the chip's eight
// dies has a run of tiles of its own, and its workgroups take neighbours at the same time, so that the die's L2 cache has the
// shared lines for both (256 x 28 x 28: a workgroup with a run of its own reads 1.9 times the tensors).
struct TileRun {
    long long from, to, step;
};
__device__ inline TileRun tiles_of(const NormArgs &a)
{
    const int b = blockIdx.x, grid = gridDim.x;
    if (grid & 7) return {b, a.tiles, grid};
    return {a.tiles * (b & 7) / 8 + (b >> 3), a.tiles * ((b & 7) + 1) / 8, grid >> 3};
}

// WHOLE: planes of at least one vector whose last vectors overlap, the ordinary case
template <int DT, int WT, int NW, int K, bool WHOLE>
__global__ __launch_bounds__(NW * 64) void norm_planes_fwd_kernel(NormArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, TY = NW * kNormTYW;
    __shared__ float red[NW * kNormTX * V];
    const int ty = threadIdx.x / kNormTX;
    const TileRun run = tiles_of(a);
    // the rounds of channels: k of the registers, or all that there are
    auto rounds = [&](auto &&body) {
        if constexpr (K > 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) body(k, ty + k * TY);
        } else {
            for (int c = ty; c < a.C; c += TY) body(0, c);
        }
    };
    for (long long tile = run.from; tile < run.to; tile += run.step) {
        const PlaneAt at = plane_at<V>(a, tile);
        const elem_t *x = static_cast<const elem_t *>(a.x) + at.base;
        elem_t *y = static_cast<elem_t *>(a.y) + at.base;
        uint4 raw[K > 0 ? K : 1];
        float s[V], mean[V], rstd[V];
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = 0.f;
        auto get = [&](int c) { return plane_get<DT, WHOLE>(a, x, at, c); };
        auto value = [&](int k, int c) -> uint4 {
            if constexpr (K > 0) return raw[k];
            else return get(c);
        };
        if constexpr (K > 0) rounds([&](int k, int c) { raw[k] = get(c); });
        rounds([&](int k, int c) {
            float t[V];
            unpack<DT>(value(k, c), t);
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] += t[i];
            if constexpr (K > 0) keep_packed(raw[k], s);
        });
        column_sum<V, NW>(s, red);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            mean[i] = mean_of(s[i], a);
            s[i] = 0.f;
        }
        rounds([&](int k, int c) {
            float t[V];
            unpack<DT>(value(k, c), t);
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] += c < a.C ? (t[i] - mean[i]) * (t[i] - mean[i]) : 0.f;
            if constexpr (K > 0) keep_packed(raw[k], s);
        });
        column_sum<V, NW>(s, red);
#pragma unroll
        for (int i = 0; i < V; ++i) rstd[i] = rstd_of(s[i], a);
        if (!at.on) continue;
        rounds([&](int k, int c) {
            if (c >= a.C) return;
            float t[V];
            unpack<DT>(value(k, c), t);
            const float g = load_param<WT>(a.gamma, c, 1.f), b = load_param<WT>(a.beta, c, 0.f);
#pragma unroll
            for (int i = 0; i < V; ++i) t[i] = (t[i] - mean[i]) * rstd[i] * g + b;
            plane_put<DT, WHOLE>(a, y, at, c, pack<DT>(t));
        });
        if (ty == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (own(at.p, i)) {
                    if (a.mean) a.mean[at.pos + i] = mean[i];
                    if (a.rstd) a.rstd[at.pos + i] = rstd[i];
                }
        }
    }
}

template <int DT, int WT, int NW, int K, bool WHOLE>
__global__ __launch_bounds__(NW * 64, 4) void norm_planes_bwd_kernel(NormArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, TY = NW * kNormTYW, KR = K > 0 ? K : 1;
    __shared__ float red[NW * kNormTX * 2 * V];
    const int ty = threadIdx.x / kNormTX, tx = threadIdx.x % kNormTX;
    const elem_t *X = static_cast<const elem_t *>(a.x), *DY = static_cast<const elem_t *>(a.dy);
    elem_t *DX = static_cast<elem_t *>(a.y);
    float *part = a.part ? a.part + (size_t)blockIdx.x * 2 * a.C : nullptr;
    float ag[KR], ab[KR], gk[KR];
#pragma unroll
    for (int k = 0; k < KR; ++k) {
        ag[k] = ab[k] = 0.f;
        gk[k] = load_param<WT>(a.gamma, min(ty + k * TY, a.C - 1), 1.f);
    }
    auto rounds = [&](auto &&body) {
        if constexpr (K > 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) body(k, ty + k * TY);
        } else {
            for (int c = ty; c < a.C; c += TY) body(0, c);
        }
    };
    bool first = true;
    const TileRun run = tiles_of(a);
    if (K == 0 && part && run.from >= run.to)
        for (int c = threadIdx.x; c < 2 * a.C; c += NW * 64) part[c] = 0.f;
    for (long long tile = run.from; tile < run.to; tile += run.step, first = false) {
        const PlaneAt at = plane_at<V>(a, tile);
        uint4 rx[KR], rd[KR];
        // (a gradient of zero drops what does not exist from the sums; values of X that are near their mean keep the product zero)
        auto get = [&](int k, int c) {
            rx[k] = plane_get<DT, WHOLE, true>(a, X + at.base, at, c);
            rd[k] = plane_get<DT, WHOLE>(a, DY + at.base, at, c);
        };
        if constexpr (K > 0) rounds(get);
        float mean[V], rstd[V], c12[2 * V];
        if constexpr (WHOLE) {
            load_params<XCONV_F32, V>(a.mean, Part{0, 0, V}, 0.f, mean, at.pos);
            load_params<XCONV_F32, V>(a.rstd, Part{0, 0, V}, 0.f, rstd, at.pos);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const bool there = at.on && i < at.p.hi;
                mean[i] = there ? a.mean[at.pos + i] : 0.f;
                rstd[i] = there ? a.rstd[at.pos + i] : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) c12[i] = c12[V + i] = 0.f;
        rounds([&](int k, int c) {
            if constexpr (K == 0) get(0, c);
            float x[V], d[V], sg = 0.f, sb = 0.f;
            unpack<DT>(rx[k], x);
            unpack<DT>(rd[k], d);
            const float g = K > 0 ? gk[k] : load_param<WT>(a.gamma, c, 1.f);
            if (!a.ragged) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float t = d[i] * ((x[i] - (WHOLE || c < a.C ? mean[i] : 0.f)) * rstd[i]);
                    c12[i] += d[i] * g;
                    c12[V + i] += t * g;
                    sg += t;
                    sb += d[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float t = d[i] * ((x[i] - (WHOLE || c < a.C ? mean[i] : 0.f)) * rstd[i]);
                    c12[i] += d[i] * g;
                    c12[V + i] += t * g;
                    sg += i >= at.p.lo ? t : 0.f;
                    sb += i >= at.p.lo ? d[i] : 0.f;
                }
            }
            if constexpr (K > 0) {
                ag[k] += sg;
                ab[k] += sb;
                asm volatile("" : "+v"(ag[k]), "+v"(ab[k]), "+v"(rx[k].x), "+v"(rd[k].x));
                keep_packed(rx[k], c12);
                keep_packed(rd[k], c12);
            } else if (part) {
#pragma unroll
                for (int o = kNormTX / 2; o >= 1; o >>= 1) {
                    sg += __shfl_xor(sg, o);
                    sb += __shfl_xor(sb, o);
                }
                if (tx == 0) {
                    part[c] = (first ? 0.f : part[c]) + sg;
                    part[(size_t)a.C + c] = (first ? 0.f : part[(size_t)a.C + c]) + sb;
                }
            }
        });
        if (!DX) continue;
        column_sum<2 * V, NW>(c12, red);
        if (!at.on) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            c12[i] *= a.inv_c * rstd[i];
            c12[V + i] *= a.inv_c * rstd[i] * rstd[i];
        }
        rounds([&](int k, int c) {
            if (c >= a.C) return;
            if constexpr (K == 0) get(0, c);
            float x[V], d[V];
            unpack<DT>(rx[k], x);
            unpack<DT>(rd[k], d);
            const float g = K > 0 ? gk[k] : load_param<WT>(a.gamma, c, 1.f);
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = (d[i] * (g * rstd[i]) - c12[i]) - (x[i] - mean[i]) * c12[V + i];
            plane_put<DT, WHOLE>(a, DX + at.base, at, c, pack<DT>(x));
        });
    }
    if (K == 0 || !part) return;
    rounds([&](int k, int c) {
        float sg = ag[k], sb = ab[k];
#pragma unroll
        for (int o = kNormTX / 2; o >= 1; o >>= 1) {
            sg += __shfl_xor(sg, o);
            sb += __shfl_xor(sb, o);
        }
        if (tx == 0 && c < a.C) {
            part[c] = sg;
            part[(size_t)a.C + c] = sb;
        }
    });
}

// out[c] = sum over the n workgroups' partial sums, in order: a workgroup takes 16 columns, its 64 rows of threads share the sums
constexpr int kJoinCols = 16, kJoinThreads = 1024;
template <int WT>
__global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(const float *part, int n, int C, void *dgamma, void *dbeta)
{
    constexpr int RW = kJoinThreads / kJoinCols;
    __shared__ float red[kJoinThreads / 64][kJoinCols];
    const int col = threadIdx.x % kJoinCols, w = threadIdx.x / kJoinCols;
    const long long q = (long long)blockIdx.x * kJoinCols + col;
    float s = 0.f;
    if (q < 2LL * C) {
#pragma unroll 16
        for (int b = w; b < n; b += RW) s += part[(size_t)b * 2 * C + q];
    }
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if ((threadIdx.x & 63) < kJoinCols) red[threadIdx.x >> 6][col] = s;
    __syncthreads();
    if (threadIdx.x >= kJoinCols || q >= 2LL * C) return;
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kJoinThreads / 64; ++i) t += red[i][col];
    typedef typename NormElem<WT>::t elem_t;
    elem_t *out = static_cast<elem_t *>(q < C ? dgamma : dbeta);
    if (out) out[q < C ? q : q - C] = norm_round<WT>(t);
}

// ---- launches ------------------------------------------------------------------------------------------------------
struct NormShape {
    int G, K, R;    // rows: lanes a row, vectors a lane (0: read again), rows at once
    int NW;         // planes: waves a workgroup
    int V;
};

// The smallest group that holds a row with one vector a lane; past a wave, two and four vectors a lane, then groups of several
// waves.  Few vectors a row: several rows at once, so that enough loads are under way.
NormShape rows_shape(int dtype, int C, bool backward)
{
    const int V = dtype == XCONV_F32 ? 4 : 8, nv = ceil_div(C, V);
    for (int G : {4, 8, 16, 32, 64})
        if (nv <= G) return {G, 1, backward ? 2 : 4, 0, V};
    if (nv <= 128) return {64, 2, backward ? 1 : 2, 0, V};
    if (nv <= 256) return {64, 4, 1, 0, V};
    for (int G : {256, 512, 1024})
        for (int K : {2, 3, 4})
            if (nv <= K * G && (G == 256 || K > 2) && !(backward && G == 1024 && K > 3)) return {G, K, 1, 0, V};
    return {1024, 0, 1, 0, V};
}
// 8 channels a wave and round: enough waves for 4 rounds, 8 with 16 waves
NormShape planes_shape(int dtype, int C)
{
    const int V = dtype == XCONV_F32 ? 4 : 8;
    for (int NW : {4, 8, 16})
        for (int K : {1, 2, 4})
            if (C <= kNormTYW * NW * K) return {0, K, 1, NW, V};
    if (C <= kNormTYW * 16 * 8) return {0, 8, 1, 16, V};
    return {0, 0, 1, 16, V};
}

constexpr int kNormBlocks = 1024;           // most workgroups that leave partial sums
constexpr long long kNormGrid = 1 << 20;    // most workgroups of the forward pass

long long plane_tiles(const xconv_norm_desc *d, int V) { return (d->outer * ceil_div((int)d->inner, V) + kNormTX - 1) / kNormTX; }

// workgroups of a pass: one piece of work each in the forward pass, of the backward pass at most kNormBlocks
int norm_blocks(const xconv_norm_desc *d, const NormShape &s, bool bwd)
{
    const int rows = s.G ? std::max(256, s.G) / s.G * s.R : 1;
    const long long want = d->inner > 1 ? plane_tiles(d, s.V) : (d->outer + rows - 1) / rows;
    return (int)std::min<long long>(d->inner > 1 && want > 8 ? (want + 7) / 8 * 8 : want, bwd ? kNormBlocks : kNormGrid);
}

template <int DT, int WT, int G, int K, int RF, int RB> hipError_t go_rows(const NormArgs &a, bool bwd, int blocks, hipStream_t st)
{
    constexpr int T = row_threads<G>, RP = T / G;
    if (!bwd) {
        hipLaunchKernelGGL((norm_rows_fwd_kernel<DT, WT, G, K, RF>), dim3((unsigned)blocks), dim3(T), 0, st, a);
    } else if constexpr (RB > 0) {
        const size_t lds = RP > 1 && a.part ? (size_t)RP * 2 * G * K * NormElem<DT>::V * 4 : 0;
        hipLaunchKernelGGL((norm_rows_bwd_kernel<DT, WT, G, K, RB>), dim3((unsigned)blocks), dim3(T), lds, st, a);
    }
    return hipGetLastError();
}
// (rows at once of the two passes as rows_shape says; 0: that shape is not a backward one)
template <int DT, int WT> hipError_t go_rows_shape(const NormArgs &a, const NormShape &s, bool bwd, int blocks, hipStream_t st)
{
    switch (s.G * 8 + s.K) {
    case 4 * 8 + 1: return go_rows<DT, WT, 4, 1, 4, 2>(a, bwd, blocks, st);
    case 8 * 8 + 1: return go_rows<DT, WT, 8, 1, 4, 2>(a, bwd, blocks, st);
    case 16 * 8 + 1: return go_rows<DT, WT, 16, 1, 4, 2>(a, bwd, blocks, st);
    case 32 * 8 + 1: return go_rows<DT, WT, 32, 1, 4, 2>(a, bwd, blocks, st);
    case 64 * 8 + 1: return go_rows<DT, WT, 64, 1, 4, 2>(a, bwd, blocks, st);
    case 64 * 8 + 2: return go_rows<DT, WT, 64, 2, 2, 1>(a, bwd, blocks, st);
    case 64 * 8 + 4: return go_rows<DT, WT, 64, 4, 1, 1>(a, bwd, blocks, st);
    case 256 * 8 + 2: return go_rows<DT, WT, 256, 2, 1, 1>(a, bwd, blocks, st);
    case 256 * 8 + 3: return go_rows<DT, WT, 256, 3, 1, 1>(a, bwd, blocks, st);
    case 256 * 8 + 4: return go_rows<DT, WT, 256, 4, 1, 1>(a, bwd, blocks, st);
    case 512 * 8 + 3: return go_rows<DT, WT, 512, 3, 1, 1>(a, bwd, blocks, st);
    case 512 * 8 + 4: return go_rows<DT, WT, 512, 4, 1, 1>(a, bwd, blocks, st);
    case 1024 * 8 + 3: return go_rows<DT, WT, 1024, 3, 1, 1>(a, bwd, blocks, st);
    case 1024 * 8 + 4: return go_rows<DT, WT, 1024, 4, 1, 0>(a, bwd, blocks, st);
    default: return go_rows<DT, WT, 1024, 0, 1, 1>(a, bwd, blocks, st);
    }
}
template <int DT, int WT, int NW, int K> hipError_t go_planes(const NormArgs &a, bool bwd, int blocks, hipStream_t st)
{
    const dim3 grid((unsigned)blocks), block(NW * 64);
    if (a.exact) {
        if (!bwd) hipLaunchKernelGGL((norm_planes_fwd_kernel<DT, WT, NW, K, false>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((norm_planes_bwd_kernel<DT, WT, NW, K, false>), grid, block, 0, st, a);
    } else {
        if (!bwd) hipLaunchKernelGGL((norm_planes_fwd_kernel<DT, WT, NW, K, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((norm_planes_bwd_kernel<DT, WT, NW, K, true>), grid, block, 0, st, a);
    }
    return hipGetLastError();
}
template <int DT, int WT> hipError_t go_planes_shape(const NormArgs &a, const NormShape &s, bool bwd, int blocks, hipStream_t st)
{
    switch (s.NW * 32 + s.K) {
    case 4 * 32 + 1: return go_planes<DT, WT, 4, 1>(a, bwd, blocks, st);
    case 4 * 32 + 2: return go_planes<DT, WT, 4, 2>(a, bwd, blocks, st);
    case 4 * 32 + 4: return go_planes<DT, WT, 4, 4>(a, bwd, blocks, st);
    case 8 * 32 + 4: return go_planes<DT, WT, 8, 4>(a, bwd, blocks, st);
    case 16 * 32 + 4: return go_planes<DT, WT, 16, 4>(a, bwd, blocks, st);
    case 16 * 32 + 8: return go_planes<DT, WT, 16, 8>(a, bwd, blocks, st);
    default: return go_planes<DT, WT, 16, 0>(a, bwd, blocks, st);
    }
}

bool overlap(const void *a, const void *b, size_t bytes)
{
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    return a && b && p < q + bytes && q < p + bytes;
}

template <int DT, int WT> hipError_t launch_norm_dt(const xconv_norm_desc *d, NormArgs a, bool bwd, void *dgamma, void *dbeta, hipStream_t st)
{
    const bool planes = d->inner > 1;
    constexpr int V = NormElem<DT>::V;
    // outputs over inputs: the overlapping part of a plane may be another workgroup's, that of a row read again another lane's
    const size_t bytes = (size_t)d->outer * d->C * d->inner * (DT == XCONV_F32 ? 4 : 2);
    const bool over = overlap(a.y, a.x, bytes) || overlap(a.y, a.dy, bytes);
    const NormShape s = planes ? planes_shape(DT, d->C) : rows_shape(DT, d->C, bwd);
    a.ragged = (planes ? d->inner : (int64_t)d->C) % V != 0;
    a.exact = planes ? over || d->inner < V : d->C < V || (s.K == 0 && over);
    a.outer = d->outer;
    a.C = d->C;
    a.inner = (int)d->inner;
    a.eps = d->eps;
    a.count = (float)d->C;
    a.inv_c = 1.0f / a.count;
    a.nvi = ceil_div((int)d->inner, s.V);
    a.tiles = plane_tiles(d, s.V);
    const int blocks = norm_blocks(d, s, bwd);
    hipError_t e = hipSuccess;
    if (d->outer > 0) e = planes ? go_planes_shape<DT, WT>(a, s, bwd, blocks, st) : go_rows_shape<DT, WT>(a, s, bwd, blocks, st);
    if (e != hipSuccess || !bwd || !(dgamma || dbeta)) return e;
    hipLaunchKernelGGL(norm_join_kernel<WT>, dim3((unsigned)ceil_div(2 * d->C, kJoinCols)), dim3(kJoinThreads), 0, st, a.part, blocks, d->C, dgamma, dbeta);
    return hipGetLastError();
}

hipError_t launch_norm(const xconv_norm_desc *d, const NormArgs &a, bool bwd, void *dgamma, void *dbeta, hipStream_t st)
{
    const bool w32 = d->w_dtype == XCONV_F32;
    if (d->dtype == XCONV_F32) return launch_norm_dt<XCONV_F32, XCONV_F32>(d, a, bwd, dgamma, dbeta, st);
    if (d->dtype == XCONV_BF16)
        return w32 ? launch_norm_dt<XCONV_BF16, XCONV_F32>(d, a, bwd, dgamma, dbeta, st) : launch_norm_dt<XCONV_BF16, XCONV_BF16>(d, a, bwd, dgamma, dbeta, st);
    return w32 ? launch_norm_dt<XCONV_F16, XCONV_F32>(d, a, bwd, dgamma, dbeta, st) : launch_norm_dt<XCONV_F16, XCONV_F16>(d, a, bwd, dgamma, dbeta, st);
}

}  // namespace

size_t norm_ws_bytes(const xconv_norm_desc *d)
{
    const bool planes = d->inner > 1;
    const NormShape s = planes ? planes_shape(d->dtype, d->C) : rows_shape(d->dtype, d->C, true);
    return (size_t)norm_blocks(d, s, true) * 2 * d->C * sizeof(float);
}

hipError_t launch_norm_fwd(const xconv_norm_desc *d, const void *X, const void *gamma, const void *beta, void *Y, float *mean, float *rstd, hipStream_t st)
{
    NormArgs a{};
    a.x = X; a.gamma = gamma; a.beta = beta; a.y = Y; a.mean = mean; a.rstd = rstd;
    return launch_norm(d, a, false, nullptr, nullptr, st);
}

hipError_t launch_norm_bwd(const xconv_norm_desc *d, const void *dY, const void *X, const float *mean, const float *rstd, const void *gamma, void *dX,
                           void *dgamma, void *dbeta, float *part, hipStream_t st)
{
    NormArgs a{};
    a.x = X; a.dy = dY; a.gamma = gamma; a.y = dX;
    a.mean = const_cast<float *>(mean);
    a.rstd = const_cast<float *>(rstd);
    a.part = dgamma || dbeta ? part : nullptr;
    return launch_norm(d, a, true, dgamma, dbeta, st);
}

}  // namespace xc
