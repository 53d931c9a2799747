// What the normalisations over channels share: 16-byte vectors of values of any type at any alignment, sums over the lanes of a row
// and over the channels of a tile of positions, and which part of a tensor a workgroup takes.
// A tensor is [outer, C, inner]: inner == 1 are rows (channels-last activations), inner > 1 planes.
#pragma once
#include <algorithm>

#include "common.h"

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

// A tensor [outer, C, inner] and how it is read
struct NormGeom {
    long long outer;
    int C, inner;
    float eps, inv_c, count;   // count = C, inv_c = 1 / C
    int nvi;              // vectors a plane
    long long tiles;      // tiles of kNormTX vectors of positions, or what the kernel takes (planes)
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
__device__ inline float mean_of(float s, const NormGeom &a)
{
    const float q = s * a.inv_c;
    return fabsf(q) < 1e30f ? fmaf(fmaf(-q, a.count, s), a.inv_c, q) : q;
}
__device__ inline float rstd_of(float squares, const NormGeom &a) { return rsqrtf(squares * a.inv_c + a.eps); }

// sums of R values over a group of G lanes of a wave, or of several waves of a workgroup of T threads through `red` (two slots of
// R * T / 64 floats, taken in turn so that one barrier a sum is enough)
template <int G, int R, int T = G> __device__ inline void group_sum(float (&s)[R], float *red, int &turn)
{
#pragma unroll
    for (int o = (G < 64 ? G : 64) / 2; o >= 1; o >>= 1)
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] += __shfl_xor(s[r], o);
    if constexpr (G > 64) {
        constexpr int W = G / 64;
        float *slot = red + turn * (T / 64) * R;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int r = 0; r < R; ++r) slot[(threadIdx.x >> 6) * R + r] = s[r];
        __syncthreads();
        if constexpr (T > G) slot += threadIdx.x / G * W * R;
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
template <int G> __device__ inline bool masked(const NormGeom &a, int k, int nv)
{
    if constexpr (G <= 64) return a.ragged;
    else return a.ragged && __builtin_amdgcn_readfirstlane((int)(threadIdx.x % G) | 63) + k * G >= nv - 1;
}

template <int G> constexpr int row_threads = G > 256 ? G : 256;

// ---- planes --------------------------------------------------------------------------------------------------------
constexpr int kNormTX = 8;               // lanes along the positions
constexpr int kNormTYW = 64 / kNormTX;   // channels of a wave

// sums over the threads along the channels of N columns of V positions each, TX lanes lie along the positions; `red` [NW][TX][N * V].
// FRESH: nobody still reads `red` (the caller takes two in turn)
template <int N, int NW, int TX = kNormTX, bool FRESH = false> __device__ inline void column_sum(float (&s)[N], float *red)
{
#pragma unroll
    for (int o = TX; o < 64; o <<= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += __shfl_xor(s[i], o);
    const int tx = threadIdx.x % TX;
    if constexpr (!FRESH) __syncthreads();   // whoever still reads the last sum
    if ((threadIdx.x & 63) < TX)
#pragma unroll
        for (int i = 0; i < N; ++i) red[((threadIdx.x >> 6) * TX + tx) * N + i] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = 0.f;
#pragma unroll 2
    for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += red[(w * TX + tx) * N + i];
}

// where the thread's vector of positions lies: first value of channel 0 of the image, its first position, the vector's part
struct PlaneAt {
    size_t base;
    long long pos;
    Part p;
    bool on;
};
template <int V, int TX = kNormTX> __device__ inline PlaneAt plane_at(const NormGeom &a, long long tile)
{
    const long long q = tile * TX + threadIdx.x % TX;
    const long long img = a.tiles * TX < (1LL << 31) ? (long long)((uint32_t)q / (uint32_t)a.nvi) : q / a.nvi;
    if (img >= a.outer) return {0, 0, {0, 0, V}, false};
    const Part p = part_of<V>((int)(q - img * a.nvi), a.inner, a.exact);
    return {(size_t)img * a.C * a.inner, img * a.inner + p.at, p, true};
}
// channel c of the vector; WHOLE: the planes are whole or overlapping vectors, and every lane loads (where there is nothing: zeros, or
// with ANY the values of another channel or position)
template <int DT, bool WHOLE, bool ANY = false> __device__ inline uint4 plane_get(const NormGeom &a, const typename NormElem<DT>::t *x, const PlaneAt &at, int c)
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
template <int DT, bool WHOLE> __device__ inline void plane_put(const NormGeom &a, typename NormElem<DT>::t *y, const PlaneAt &at, int c, const uint4 &v)
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
__device__ inline TileRun tiles_of(const NormGeom &a)
{
    const int b = blockIdx.x, grid = gridDim.x;
    if (grid & 7) return {b, a.tiles, grid};
    return {a.tiles * (b & 7) / 8 + (b >> 3), a.tiles * ((b & 7) + 1) / 8, grid >> 3};
}

// ---- host ----------------------------------------------------------------------------------------------------------
inline long long plane_tiles(const xconv_norm_desc *d, int V, int TX = kNormTX) { return (d->outer * ceil_div((int)d->inner, V) + TX - 1) / TX; }

inline bool overlap(const void *a, const void *b, size_t bytes)
{
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    return a && b && p < q + bytes && q < p + bytes;
}

}  // namespace

}  // namespace xc
