// Layer normalisation over the channels of every position, forward and backward.
//     forward   mean = sum_c x / C, var = sum_c (x - mean)^2 / C, rstd = 1 / sqrt(var + eps), y = (x - mean) rstd gamma + beta
//     backward  g = dy gamma, xh = (x - mean) rstd, dx = rstd (g - sum_c g / C - xh sum_c (g xh) / C),
//               dgamma = sum over positions of dy xh, dbeta = sum over positions of dy
// X is [outer, C, inner]: inner == 1 are rows (channels-last activations), inner > 1 planes.  Sums are fp32; the variance is
// summed from the centred values (a mean far from zero costs no digits), every output is rounded once.
// Bound by HBM: every tensor is read once, its values stay in registers between the statistics and the output.
//
// Rows: a group of G lanes (part of a wave, a wave, or a workgroup) holds a row, K 16-byte vectors a lane, and sums across
// lanes.  Planes: 16 lanes lie along the positions (256 consecutive bytes of a plane), the other threads along the channels,
// K channels each; sums across threads go through LDS.  Longer rows and more channels than the registers hold are read
// again from the cache (K == 0).  Rows of any length are read as vectors at the alignment of an element, which the memory
// system takes; only the last vector of a row or plane is read value by value.
//
// Backward: a fixed number of workgroups walks the positions and adds up dgamma and dbeta in registers, in fixed order; their
// partial sums are added up in order by a second launch, so that results do not depend on timing.
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

// the first n (1 .. V) values of a vector; the others are zero / left alone
template <int DT> __device__ inline uint4 load_some(const typename NormElem<DT>::t *p, int n)
{
    constexpr int V = NormElem<DT>::V;
    if (n >= V) return load_loose<DT>(p);
    typename NormElem<DT>::t e[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = i < n ? p[i] : typename NormElem<DT>::t(0);
    return __builtin_bit_cast(uint4, e);
}
template <int DT> __device__ inline void store_some(typename NormElem<DT>::t *p, const uint4 &v, int n)
{
    constexpr int V = NormElem<DT>::V;
    if (n >= V) {
        store_loose<DT>(p, v);
        return;
    }
    struct Pack { typename NormElem<DT>::t e[V]; };
    const Pack k = __builtin_bit_cast(Pack, v);
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < n) p[i] = k.e[i];
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
        else w[i] = (uint32_t)f32_to_st16<DT>(x[2 * i]) | (uint32_t)f32_to_st16<DT>(x[2 * i + 1]) << 16;
    }
    return uint4{w[0], w[1], w[2], w[3]};
}
// V parameters from channel c on (n of them exist), in the type WT
template <int WT, int V> __device__ inline void load_params(const void *p, int c, int n, float none, float (&out)[V])
{
    typedef typename NormElem<WT>::t elem_t;
    const elem_t *q = static_cast<const elem_t *>(p) + c;
    constexpr int VW = NormElem<WT>::V;
    if (!p) {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = none;
    } else if (n >= V && V >= VW) {
#pragma unroll
        for (int j = 0; j < V; j += VW) {
            float t[VW];
            unpack<WT>(load_loose<WT>(q + j), t);
#pragma unroll
            for (int i = 0; i < VW; ++i) out[j + i] = t[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = i < n ? norm_val<WT>(q[i]) : none;
    }
}
template <int WT> __device__ inline float load_param(const void *p, int c, float none)
{
    return p ? norm_val<WT>(static_cast<const typename NormElem<WT>::t *>(p)[c]) : none;
}

// sum over a group of G lanes of a wave, or over the workgroup's G threads through `red` (two slots of G / 64 floats, taken in
// turn so that one barrier a sum is enough)
template <int G> __device__ inline float group_sum(float s, float *red, int &turn)
{
#pragma unroll
    for (int o = (G < 64 ? G : 64) / 2; o >= 1; o >>= 1) s += __shfl_xor(s, o);
    if constexpr (G > 64) {
        constexpr int W = G / 64;
        float *slot = red + turn * W;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = s;
        __syncthreads();
        s = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) s += slot[i];
    }
    return s;
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
    long long tiles;      // tiles of 16 vectors of positions (planes)
};

// ---- rows ----------------------------------------------------------------------------------------------------------
// G lanes a row, K vectors a lane (lane l holds vectors l, l + G, ...); K == 0: the row is read once a pass.
template <int DT, int WT, int G, int K>
__global__ __launch_bounds__(G > 256 ? G : 256) void norm_rows_fwd_kernel(NormArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, T = G > 256 ? G : 256, RP = T / G;
    __shared__ float red[G > 64 ? 2 * (G / 64) : 1];
    int turn = 0;
    const int lane = threadIdx.x % G;
    const int nv = (a.C + V - 1) / V;
    auto left = [&](int v) { return a.C - v * V; };
    for (long long r0 = (long long)blockIdx.x * RP; r0 < a.outer; r0 += (long long)gridDim.x * RP) {   // (the same count for all threads)
        const long long row = r0 + threadIdx.x / G;
        const bool on = row < a.outer;
        const elem_t *x = static_cast<const elem_t *>(a.x) + (size_t)(on ? row : 0) * a.C;
        elem_t *y = static_cast<elem_t *>(a.y) + (size_t)(on ? row : 0) * a.C;
        uint4 raw[K > 0 ? K : 1];
        // the rounds of vectors: k of the registers, or all that there are
        auto rounds = [&](auto &&body) {
            if constexpr (K > 0) {
#pragma unroll
                for (int k = 0; k < K; ++k) body(k, lane + k * G);
            } else {
                for (int v = lane; v < nv; v += G) body(0, v);
            }
        };
        if constexpr (K > 0) rounds([&](int k, int v) { raw[k] = v < nv ? load_some<DT>(x + v * V, left(v)) : uint4{0, 0, 0, 0}; });
        auto value = [&](int k, int v) -> uint4 {
            if constexpr (K > 0) return raw[k];
            else return load_some<DT>(x + v * V, left(v));
        };
        float s = 0.f;
        rounds([&](int k, int v) {
            float t[V];
            unpack<DT>(value(k, v), t);
#pragma unroll
            for (int i = 0; i < V; ++i) s += t[i];
        });
        const float mean = group_sum<G>(s, red, turn) / a.count;
        s = 0.f;
        rounds([&](int k, int v) {
            const int n = left(v);
            float t[V];
            unpack<DT>(value(k, v), t);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = i < n ? t[i] - mean : 0.f;
                s += d * d;
            }
        });
        const float rstd = 1.0f / sqrtf(group_sum<G>(s, red, turn) * a.inv_c + a.eps);
        if (!on) continue;
        rounds([&](int k, int v) {
            if (v >= nv) return;
            float t[V], g[V], b[V];
            unpack<DT>(value(k, v), t);
            load_params<WT, V>(a.gamma, v * V, left(v), 1.f, g);
            load_params<WT, V>(a.beta, v * V, left(v), 0.f, b);
#pragma unroll
            for (int i = 0; i < V; ++i) t[i] = (t[i] - mean) * rstd * g[i] + b[i];
            store_some<DT>(y + v * V, pack<DT>(t), left(v));
        });
        if (lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// A workgroup's groups walk the rows; every lane adds up dgamma and dbeta of its own columns.  K == 0: one row a workgroup at
// a time, dgamma and dbeta in the workgroup's own slots of `part`.
template <int DT, int WT, int G, int K>
__global__ __launch_bounds__(G > 256 ? G : 256) void norm_rows_bwd_kernel(NormArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, T = G > 256 ? G : 256, RP = T / G;
    __shared__ float red[G > 64 ? 2 * (G / 64) : 1];
    int turn = 0;
    const int lane = threadIdx.x % G, grp = threadIdx.x / G;
    const elem_t *X = static_cast<const elem_t *>(a.x), *DY = static_cast<const elem_t *>(a.dy);
    elem_t *DX = static_cast<elem_t *>(a.y);
    const int nv = (a.C + V - 1) / V;
    auto left = [&](int v) { return a.C - v * V; };
    float *part = a.part ? a.part + (size_t)blockIdx.x * 2 * a.C : nullptr;
    if constexpr (K > 0) {
        float g[K][V], ag[K][V], ab[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int v = lane + k * G;
            load_params<WT, V>(a.gamma, v * V, left(v), 1.f, g[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) ag[k][i] = ab[k][i] = 0.f;
        }
        for (long long r0 = (long long)blockIdx.x * RP; r0 < a.outer; r0 += (long long)gridDim.x * RP) {   // (the same count for all threads)
            const long long row = r0 + grp;
            const bool on = row < a.outer;
            const size_t at = (size_t)(on ? row : 0) * a.C;
            const float mean = a.mean[on ? row : 0], rstd = a.rstd[on ? row : 0];
            uint4 rx[K], rd[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int v = lane + k * G;
                const bool has = on && v < nv;
                rx[k] = has ? load_some<DT>(X + at + v * V, left(v)) : uint4{0, 0, 0, 0};
                rd[k] = has ? load_some<DT>(DY + at + v * V, left(v)) : uint4{0, 0, 0, 0};
            }
            float c1 = 0.f, c2 = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float x[V], d[V];
                unpack<DT>(rx[k], x);
                unpack<DT>(rd[k], d);
                const int n = on ? left(lane + k * G) : 0;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xh = i < n ? (x[i] - mean) * rstd : 0.f, gd = i < n ? d[i] * g[k][i] : 0.f;
                    c1 += gd;
                    c2 += gd * xh;
                    ag[k][i] += d[i] * xh;
                    ab[k][i] += d[i];
                }
            }
            c1 = group_sum<G>(c1, red, turn) * a.inv_c;
            c2 = group_sum<G>(c2, red, turn) * a.inv_c;
            if (DX && on) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const int v = lane + k * G;
                    if (v >= nv) continue;
                    float x[V], d[V];
                    unpack<DT>(rx[k], x);
                    unpack<DT>(rd[k], d);
#pragma unroll
                    for (int i = 0; i < V; ++i) x[i] = rstd * (d[i] * g[k][i] - c1 - (x[i] - mean) * rstd * c2);
                    store_some<DT>(DX + at + v * V, pack<DT>(x), left(v));
                }
            }
        }
        if (!part) return;
        // groups of one workgroup hold the same columns: added up in order of the groups
        if constexpr (RP > 1) {
            extern __shared__ float cols[];     // [RP][2][G * K * V]
            constexpr int W = G * K * V;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = (lane + k * G) * V + i;
                    cols[(grp * 2) * W + c] = ag[k][i];
                    cols[(grp * 2 + 1) * W + c] = ab[k][i];
                }
            __syncthreads();
            for (int q = threadIdx.x; q < 2 * W; q += T) {
                const int c = q % W;
                if (c >= a.C) continue;
                float s = 0.f;
                for (int r = 0; r < RP; ++r) s += cols[r * 2 * W + q];
                part[(size_t)(q / W) * a.C + c] = s;
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = (lane + k * G) * V + i;
                    if (c < a.C) {
                        part[c] = ag[k][i];
                        part[(size_t)a.C + c] = ab[k][i];
                    }
                }
        }
    } else {
        bool first = true;
        for (long long row = blockIdx.x; row < a.outer; row += gridDim.x, first = false) {
            const size_t at = (size_t)row * a.C;
            const float mean = a.mean[row], rstd = a.rstd[row];
            float c1 = 0.f, c2 = 0.f;
            for (int v = lane; v < nv; v += G) {
                float x[V], d[V], g[V];
                unpack<DT>(load_some<DT>(X + at + v * V, left(v)), x);
                unpack<DT>(load_some<DT>(DY + at + v * V, left(v)), d);
                load_params<WT, V>(a.gamma, v * V, left(v), 1.f, g);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xh = i < left(v) ? (x[i] - mean) * rstd : 0.f, gd = i < left(v) ? d[i] * g[i] : 0.f;
                    c1 += gd;
                    c2 += gd * xh;
                    if (part && i < left(v)) {
                        float *pg = part + v * V + i, *pb = pg + a.C;
                        *pg = (first ? 0.f : *pg) + d[i] * xh;
                        *pb = (first ? 0.f : *pb) + d[i];
                    }
                }
            }
            c1 = group_sum<G>(c1, red, turn) * a.inv_c;
            c2 = group_sum<G>(c2, red, turn) * a.inv_c;
            if (!DX) continue;
            for (int v = lane; v < nv; v += G) {
                float x[V], d[V], g[V];
                unpack<DT>(load_some<DT>(X + at + v * V, left(v)), x);
                unpack<DT>(load_some<DT>(DY + at + v * V, left(v)), d);
                load_params<WT, V>(a.gamma, v * V, left(v), 1.f, g);
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = rstd * (d[i] * g[i] - c1 - (x[i] - mean) * rstd * c2);
                store_some<DT>(DX + at + v * V, pack<DT>(x), left(v));
            }
        }
    }
}

// ---- planes --------------------------------------------------------------------------------------------------------
constexpr int kNormTX = 16;     // lanes along the positions

// sums over the TY threads of each of the 16 columns of vectors, V positions each; `red` [NW][16][V]
template <int V, int NW> __device__ inline void column_sum(float (&s)[V], float *red)
{
#pragma unroll
    for (int i = 0; i < V; ++i) {
        s[i] += __shfl_xor(s[i], 16);
        s[i] += __shfl_xor(s[i], 32);
    }
    const int tx = threadIdx.x % kNormTX;
    __syncthreads();                     // whoever still reads the last sum
    if ((threadIdx.x & 63) < kNormTX)
#pragma unroll
        for (int i = 0; i < V; ++i) red[((threadIdx.x >> 6) * kNormTX + tx) * V + i] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] += red[(w * kNormTX + tx) * V + i];
}

// where the thread's vector of positions lies: first value of channel 0, values that exist (0: past the end), first position
struct PlaneAt {
    size_t base;
    long long pos;
    int n;
};
template <int V> __device__ inline PlaneAt plane_at(const NormArgs &a, long long tile)
{
    const long long q = tile * kNormTX + threadIdx.x % kNormTX;
    const long long img = q / a.nvi;
    if (img >= a.outer) return {0, 0, 0};
    const int p = (int)(q - img * a.nvi) * V;
    return {(size_t)img * a.C * a.inner + p, img * a.inner + p, min(V, a.inner - p)};
}

template <int DT, int WT, int NW, int K>
__global__ __launch_bounds__(NW * 64) void norm_planes_fwd_kernel(NormArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, TY = NW * 4;
    __shared__ float red[NW * kNormTX * V];
    const int ty = threadIdx.x / kNormTX;
    for (long long tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const PlaneAt at = plane_at<V>(a, tile);
        const elem_t *x = static_cast<const elem_t *>(a.x) + at.base;
        elem_t *y = static_cast<elem_t *>(a.y) + at.base;
        const bool on = at.n > 0;
        uint4 raw[K > 0 ? K : 1];
        float s[V], mean[V], rstd[V];
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = 0.f;
        // the rounds of channels: k of the registers, or all that there are
        auto rounds = [&](auto &&body) {
            if constexpr (K > 0) {
#pragma unroll
                for (int k = 0; k < K; ++k) body(k, ty + k * TY);
            } else {
                for (int c = ty; c < a.C; c += TY) body(0, c);
            }
        };
        auto value = [&](int k, int c) -> uint4 {
            if constexpr (K > 0) return raw[k];
            else return on ? load_some<DT>(x + (size_t)c * a.inner, at.n) : uint4{0, 0, 0, 0};
        };
        if constexpr (K > 0)
            rounds([&](int k, int c) { raw[k] = on && c < a.C ? load_some<DT>(x + (size_t)c * a.inner, at.n) : uint4{0, 0, 0, 0}; });
        rounds([&](int k, int c) {
            float t[V];
            unpack<DT>(value(k, c), t);
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] += t[i];
        });
        column_sum<V, NW>(s, red);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            mean[i] = s[i] / a.count;
            s[i] = 0.f;
        }
        rounds([&](int k, int c) {
            float t[V];
            unpack<DT>(value(k, c), t);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = c < a.C ? t[i] - mean[i] : 0.f;
                s[i] += d * d;
            }
        });
        column_sum<V, NW>(s, red);
#pragma unroll
        for (int i = 0; i < V; ++i) rstd[i] = 1.0f / sqrtf(s[i] * a.inv_c + a.eps);
        if (!on) continue;
        rounds([&](int k, int c) {
            if (c >= a.C) return;
            float t[V];
            unpack<DT>(value(k, c), t);
            const float g = load_param<WT>(a.gamma, c, 1.f), b = load_param<WT>(a.beta, c, 0.f);
#pragma unroll
            for (int i = 0; i < V; ++i) t[i] = (t[i] - mean[i]) * rstd[i] * g + b;
            store_some<DT>(y + (size_t)c * a.inner, pack<DT>(t), at.n);
        });
        if (ty == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < at.n) {
                    if (a.mean) a.mean[at.pos + i] = mean[i];
                    if (a.rstd) a.rstd[at.pos + i] = rstd[i];
                }
        }
    }
}

template <int DT, int WT, int NW, int K>
__global__ __launch_bounds__(NW * 64) void norm_planes_bwd_kernel(NormArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, TY = NW * 4, KR = K > 0 ? K : 1;
    __shared__ float red[NW * kNormTX * V];
    const int ty = threadIdx.x / kNormTX, tx = threadIdx.x % kNormTX;
    const elem_t *X = static_cast<const elem_t *>(a.x), *DY = static_cast<const elem_t *>(a.dy);
    elem_t *DX = static_cast<elem_t *>(a.y);
    float *part = a.part ? a.part + (size_t)blockIdx.x * 2 * a.C : nullptr;
    float ag[KR], ab[KR];
#pragma unroll
    for (int k = 0; k < KR; ++k) ag[k] = ab[k] = 0.f;
    auto rounds = [&](auto &&body) {
        if constexpr (K > 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) body(k, ty + k * TY);
        } else {
            for (int c = ty; c < a.C; c += TY) body(0, c);
        }
    };
    bool first = true;
    for (long long tile = blockIdx.x; tile < a.tiles; tile += gridDim.x, first = false) {
        const PlaneAt at = plane_at<V>(a, tile);
        const bool on = at.n > 0;
        uint4 rx[KR], rd[KR];
        auto get = [&](const elem_t *t, int c) { return on && c < a.C ? load_some<DT>(t + at.base + (size_t)c * a.inner, at.n) : uint4{0, 0, 0, 0}; };
        if constexpr (K > 0) rounds([&](int k, int c) { rx[k] = get(X, c); rd[k] = get(DY, c); });
        float mean[V], rstd[V], c1[V], c2[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            mean[i] = i < at.n ? a.mean[at.pos + i] : 0.f;
            rstd[i] = i < at.n ? a.rstd[at.pos + i] : 0.f;
            c1[i] = c2[i] = 0.f;
        }
        rounds([&](int k, int c) {
            if constexpr (K == 0) { rx[0] = get(X, c); rd[0] = get(DY, c); }
            float x[V], d[V], sg = 0.f, sb = 0.f;
            unpack<DT>(rx[k], x);
            unpack<DT>(rd[k], d);
            const float g = c < a.C ? load_param<WT>(a.gamma, c, 1.f) : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (x[i] - mean[i]) * rstd[i], gd = d[i] * g;
                c1[i] += gd;
                c2[i] += gd * xh;
                sg += d[i] * xh;
                sb += d[i];
            }
            if constexpr (K > 0) {
                ag[k] += sg;
                ab[k] += sb;
            } else if (part) {
#pragma unroll
                for (int o = 8; o >= 1; o >>= 1) {
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
        column_sum<V, NW>(c1, red);
        column_sum<V, NW>(c2, red);
        if (!on) continue;
        rounds([&](int k, int c) {
            if (c >= a.C) return;
            if constexpr (K == 0) { rx[0] = get(X, c); rd[0] = get(DY, c); }
            float x[V], d[V];
            unpack<DT>(rx[k], x);
            unpack<DT>(rd[k], d);
            const float g = load_param<WT>(a.gamma, c, 1.f);
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = rstd[i] * (d[i] * g - c1[i] * a.inv_c - (x[i] - mean[i]) * rstd[i] * (c2[i] * a.inv_c));
            store_some<DT>(DX + at.base + (size_t)c * a.inner, pack<DT>(x), at.n);
        });
    }
    if constexpr (K > 0) {
        if (!part) return;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float sg = ag[k], sb = ab[k];
#pragma unroll
            for (int o = 8; o >= 1; o >>= 1) {
                sg += __shfl_xor(sg, o);
                sb += __shfl_xor(sb, o);
            }
            const int c = ty + k * TY;
            if (tx == 0 && c < a.C) {
                part[c] = sg;
                part[(size_t)a.C + c] = sb;
            }
        }
    }
}

// out[c] = sum over the n workgroups' partial sums, in order: 64 columns a workgroup, its four waves share the workgroups
template <int WT>
__global__ __launch_bounds__(kThreads) void norm_join_kernel(const float *part, int n, int C, void *dgamma, void *dbeta)
{
    __shared__ float red[kThreads];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, q = blockIdx.x * 64 + lane;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (q < 2 * C) {
        int b = w;
        for (; b + 12 < n; b += 16)
#pragma unroll
            for (int u = 0; u < 4; ++u) s[u] += part[(size_t)(b + 4 * u) * 2 * C + q];
        for (; b < n; b += 4) s[0] += part[(size_t)b * 2 * C + q];
    }
    red[threadIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (w != 0 || q >= 2 * C) return;
    const float t = (red[lane] + red[64 + lane]) + (red[128 + lane] + red[192 + lane]);
    typedef typename NormElem<WT>::t elem_t;
    elem_t *out = static_cast<elem_t *>(q < C ? dgamma : dbeta);
    if (out) out[q < C ? q : q - C] = norm_round<WT>(t);
}

// ---- launches ------------------------------------------------------------------------------------------------------
struct NormShape {
    int G, K;       // rows: lanes a row, vectors a lane (0: read again)
    int NW;         // planes: waves a workgroup
    int V;
};

// The smallest group that holds a row with one vector a lane; past a wave, two and four vectors a lane (more would spill the
// backward pass's sums), then groups of several waves.
NormShape rows_shape(int dtype, int C)
{
    const int V = dtype == XCONV_F32 ? 4 : 8, nv = ceil_div(C, V);
    for (int G : {4, 8, 16, 32, 64})
        if (nv <= G) return {G, 1, 0, V};
    if (nv <= 128) return {64, 2, 0, V};
    if (nv <= 256) return {64, 4, 0, V};
    for (int G : {256, 512, 1024})
        if (nv <= 2 * G) return {G, 2, 0, V};
    if (nv <= 4096) return {1024, 4, 0, V};
    return {1024, 0, 0, V};
}
// 4 channels a wave and round: enough waves for 8 rounds, then 16 rounds in the forward pass (the backward pass holds two tensors)
NormShape planes_shape(int dtype, int C, bool backward)
{
    const int V = dtype == XCONV_F32 ? 4 : 8;
    for (int NW : {4, 8, 16})
        for (int K : {1, 2, 4, 8})
            if (C <= 4 * NW * K) return {0, K, NW, V};
    if (!backward && C <= 1024) return {0, 16, 16, V};
    return {0, 0, 16, V};
}

constexpr long long kNormGrid = 1 << 20;   // most workgroups of the forward pass
constexpr int kNormBlocks = 1024;   // most workgroups that leave partial sums

int bwd_blocks(const xconv_norm_desc *d, const NormShape &s, bool planes)
{
    const long long want = planes ? (d->outer * ceil_div((int)d->inner, s.V) + kNormTX - 1) / kNormTX
                                  : (d->outer + std::max(1, 256 / std::max(1, s.G)) - 1) / std::max(1, 256 / std::max(1, s.G));
    return (int)std::min<long long>(want, kNormBlocks);
}

template <int DT, int WT, int G, int K> hipError_t go_rows(const NormArgs &a, bool bwd, int blocks, hipStream_t st)
{
    constexpr int T = G > 256 ? G : 256, RP = T / G;
    if (!bwd) {
        const long long grid = (a.outer + RP - 1) / RP;
        hipLaunchKernelGGL((norm_rows_fwd_kernel<DT, WT, G, K>), dim3((unsigned)std::min<long long>(grid, kNormGrid)), dim3(T), 0, st, a);
    } else {
        const size_t lds = RP > 1 && a.part ? (size_t)RP * 2 * G * K * NormElem<DT>::V * 4 : 0;
        hipLaunchKernelGGL((norm_rows_bwd_kernel<DT, WT, G, K>), dim3((unsigned)blocks), dim3(T), lds, st, a);
    }
    return hipGetLastError();
}
template <int DT, int WT> hipError_t go_rows_shape(const NormArgs &a, const NormShape &s, bool bwd, int blocks, hipStream_t st)
{
    switch (s.G * 8 + s.K) {
    case 4 * 8 + 1: return go_rows<DT, WT, 4, 1>(a, bwd, blocks, st);
    case 8 * 8 + 1: return go_rows<DT, WT, 8, 1>(a, bwd, blocks, st);
    case 16 * 8 + 1: return go_rows<DT, WT, 16, 1>(a, bwd, blocks, st);
    case 32 * 8 + 1: return go_rows<DT, WT, 32, 1>(a, bwd, blocks, st);
    case 64 * 8 + 1: return go_rows<DT, WT, 64, 1>(a, bwd, blocks, st);
    case 64 * 8 + 2: return go_rows<DT, WT, 64, 2>(a, bwd, blocks, st);
    case 64 * 8 + 4: return go_rows<DT, WT, 64, 4>(a, bwd, blocks, st);
    case 256 * 8 + 2: return go_rows<DT, WT, 256, 2>(a, bwd, blocks, st);
    case 512 * 8 + 2: return go_rows<DT, WT, 512, 2>(a, bwd, blocks, st);
    case 1024 * 8 + 2: return go_rows<DT, WT, 1024, 2>(a, bwd, blocks, st);
    case 1024 * 8 + 4: return go_rows<DT, WT, 1024, 4>(a, bwd, blocks, st);
    default: return go_rows<DT, WT, 1024, 0>(a, bwd, blocks, st);
    }
}
template <int DT, int WT, int NW, int K> hipError_t go_planes(const NormArgs &a, bool bwd, int blocks, hipStream_t st)
{
    if (!bwd) hipLaunchKernelGGL((norm_planes_fwd_kernel<DT, WT, NW, K>), dim3((unsigned)std::min<long long>(a.tiles, kNormGrid)), dim3(NW * 64), 0, st, a);
    else if constexpr (K <= 8) hipLaunchKernelGGL((norm_planes_bwd_kernel<DT, WT, NW, K>), dim3((unsigned)blocks), dim3(NW * 64), 0, st, a);
    return hipGetLastError();
}
template <int DT, int WT> hipError_t go_planes_shape(const NormArgs &a, const NormShape &s, bool bwd, int blocks, hipStream_t st)
{
    switch (s.NW * 32 + s.K) {
    case 4 * 32 + 1: return go_planes<DT, WT, 4, 1>(a, bwd, blocks, st);
    case 4 * 32 + 2: return go_planes<DT, WT, 4, 2>(a, bwd, blocks, st);
    case 4 * 32 + 4: return go_planes<DT, WT, 4, 4>(a, bwd, blocks, st);
    case 4 * 32 + 8: return go_planes<DT, WT, 4, 8>(a, bwd, blocks, st);
    case 8 * 32 + 8: return go_planes<DT, WT, 8, 8>(a, bwd, blocks, st);
    case 16 * 32 + 8: return go_planes<DT, WT, 16, 8>(a, bwd, blocks, st);
    case 16 * 32 + 16: return go_planes<DT, WT, 16, 16>(a, bwd, blocks, st);
    default: return go_planes<DT, WT, 16, 0>(a, bwd, blocks, st);
    }
}

template <int DT, int WT> hipError_t launch_norm_dt(const xconv_norm_desc *d, NormArgs a, bool bwd, void *dgamma, void *dbeta, hipStream_t st)
{
    const bool planes = d->inner > 1;
    const NormShape s = planes ? planes_shape(DT, d->C, bwd) : rows_shape(DT, d->C);
    a.outer = d->outer;
    a.C = d->C;
    a.inner = (int)d->inner;
    a.eps = d->eps;
    a.count = (float)d->C;
    a.inv_c = 1.0f / a.count;
    a.nvi = ceil_div((int)d->inner, s.V);
    a.tiles = (d->outer * a.nvi + kNormTX - 1) / kNormTX;
    const int blocks = bwd ? bwd_blocks(d, s, planes) : 0;
    hipError_t e = hipSuccess;
    if (d->outer > 0) e = planes ? go_planes_shape<DT, WT>(a, s, bwd, blocks, st) : go_rows_shape<DT, WT>(a, s, bwd, blocks, st);
    if (e != hipSuccess || !a.part) return e;
    hipLaunchKernelGGL(norm_join_kernel<WT>, dim3((unsigned)ceil_div(2 * d->C, 64)), dim3(kThreads), 0, st, a.part, blocks, d->C, dgamma, dbeta);
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
    const NormShape s = planes ? planes_shape(d->dtype, d->C, true) : rows_shape(d->dtype, d->C);
    return (size_t)bwd_blocks(d, s, planes) * 2 * d->C * sizeof(float);
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
