// Rows of a table by index, and the gradient of the table.
//     lookup    y_i = scale W[t_i]
//     gradient  dW_v = scale * sum over the places i with t_i = v of dy_i, in order of the places; rows that no place names are zeros
// Bound by HBM: the lookup reads the rows that are named and writes y, the gradient reads dy and writes dW.
//
// The gradient goes by the places sorted by index (stable, so the sums do not depend on timing; no float atomics).  The sort is of its
// own: an index belongs to bucket t % NB (neighbouring rows are often alike in frequency), and a workgroup counts and places the
// indices of one bucket, its 16 waves each a part of the list in order, with counters of their own for every row of the bucket.  Short
// lists are read whole by every workgroup (one launch) where 256 buckets do for the table; others are split into buckets first, the same way,
// by slices of the list.
// Sums: the sorted places in chunks of equal length, a group of lanes each; a run of equal indices that ends inside its chunk is written
// to dW, the parts of one that crosses chunks are left as floats and added in order by a last launch.  Small gradients take one launch.
//
// Measured: lookup, 131072 places of 64 fp32 from a table of 1024 rows 10.3 us (a fill of the 33.5 MB that it writes: 6.7); gradient, 65536 places of
// 512 bf16 by frequencies as in texts into 50304 rows 53 us: counting 4 us, splitting 8, sorting the buckets 8, sums and rows of zeros 24 =
// 5.0 TB/s, joining 7.  (Zeros written by the workgroups that sort the buckets: these 14, sums 20.)
#include <algorithm>

#include "launch.h"
#include "norm_core.h"

namespace xc {

namespace {

// ---- lookup --------------------------------------------------------------------------------------------------------
struct LookupArgs {
    const void *idx, *w;
    void *y;
    long long n;          // places
    long long rows;       // of the table
    int C, wide;          // wide: 64-bit indices
    float scale;
};
__device__ inline long long index_at(const void *idx, int wide, long long i)
{
    return wide ? static_cast<const long long *>(idx)[i] : (long long)static_cast<const int *>(idx)[i];
}

// G lanes a place; an index outside the table gives a row of NaN
template <int DT, int G, int R>
__global__ __launch_bounds__(kThreads) void embed_lookup_kernel(LookupArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V;
    const int lane = threadIdx.x % G, nv = (a.C + V - 1) / V, exact = a.C < V;
    constexpr int RP = kThreads / G;     // places of a workgroup, R times
    for (long long i0 = (long long)blockIdx.x * (RP * R) + threadIdx.x / G; i0 < a.n; i0 += (long long)gridDim.x * (RP * R)) {
        long long t[R];
#pragma unroll
        for (int r = 0; r < R; ++r) t[r] = i0 + r * RP < a.n ? index_at(a.idx, a.wide, i0 + r * RP) : -1;
        for (int v = blockIdx.y * G + lane; v < nv; v += gridDim.y * G) {
            const Part p = part_of<V>(v, a.C, exact);
            uint4 raw[R];
#pragma unroll
            for (int r = 0; r < R; ++r)
                raw[r] = t[r] >= 0 && t[r] < a.rows ? load_part<DT>(static_cast<const elem_t *>(a.w) + (size_t)t[r] * a.C, p) : uint4{0, 0, 0, 0};
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (i0 + r * RP >= a.n) break;
                float x[V];
                unpack<DT>(raw[r], x);
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    x[k] = t[r] >= 0 && t[r] < a.rows ? x[k] * a.scale : __builtin_nanf("");
                    // (an fp32 product that is then rounded, in every type; left alone, products become fp16 numbers in one instruction)
                    if constexpr (DT == XCONV_F16) asm("" : "+v"(x[k]));
                }
                store_part<DT>(static_cast<elem_t *>(a.y) + (size_t)(i0 + r * RP) * a.C, pack<DT>(x), p);
            }
        }
    }
}

// ---- the places in order of their indices --------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kSortKeys = 960;      // most keys of a workgroup of 16 waves: 60 KB of counters
constexpr int kSlices = 64;         // of a long list

struct SortArgs {
    const void *idx;
    int wide;
    int n;                    // places
    int rows, pad;            // of the table; the row whose places are left out (-1: none)
    int nb, shift;            // buckets, a power of two
    int slice;                // places of a slice (long lists)
    int keys;                 // most keys of a workgroup
    int *hist;                // [kSlices][nb] places of a slice and bucket
    int *first;               // [nb + 1] where the buckets begin
    int2 *split;              // index and place in order of the buckets
    int2 *sorted;             // index and place in order of bucket, index, place
    int2 *run;                // [rows] where the places of an index begin, and their number
    int *total;               // places that count
};

// kSplitList: one slice, keys are the buckets; kBucket: one bucket of a list that is split
enum SortMode { kSplitList, kBucket };

// index of place i, -1 where it does not count
__device__ inline int index_of(const SortArgs &a, int i, int end)
{
    if (i >= end) return -1;
    const long long t = index_at(a.idx, a.wide, i);
    return t >= 0 && t < a.rows && t != a.pad ? (int)t : -1;
}

// exclusive sum of s over the workgroup's threads; `sums` [waves]
__device__ inline int scan_exclusive(int s, int *sums, int &total)
{
    int in = s;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(in, o);
        if ((int)(threadIdx.x & 63) >= o) in += u;
    }
    if ((threadIdx.x & 63) == 63) sums[threadIdx.x >> 6] = in;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
        if (w < (int)(threadIdx.x >> 6)) before += sums[w];
        total += sums[w];
    }
    __syncthreads();
    return before + in - s;
}

__global__ __launch_bounds__(kSortThreads) void embed_count_kernel(SortArgs a)
{
    extern __shared__ int counts[];      // [nb]
    for (int b = threadIdx.x; b < a.nb; b += kSortThreads) counts[b] = 0;
    __syncthreads();
    const int from = blockIdx.x * a.slice, to = min(a.n, from + a.slice);
    for (int i = from + (int)threadIdx.x; i < to; i += kSortThreads) {
        const int t = index_of(a, i, to);
        if (t >= 0) atomicAdd(&counts[t & (a.nb - 1)], 1);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < a.nb; b += kSortThreads) a.hist[(size_t)blockIdx.x * a.nb + b] = counts[b];
}

// lanes whose key is the same, for keys of so many bits; none for a key below zero
__device__ inline uint64_t same_keys(int key, int bits)
{
    const uint64_t all = __ballot(key >= 0);
    uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);
    for (int b = 0; b < bits; ++b) {
        const uint32_t bit = (uint32_t)key >> b & 1u;
        const uint64_t v = __ballot(bit);
        lo &= (uint32_t)v ^ (bit - 1u);
        hi &= (uint32_t)(v >> 32) ^ (bit - 1u);
    }
    return key < 0 ? 0 : (uint64_t)hi << 32 | lo;
}
__device__ inline int lanes_below(uint64_t lanes)
{
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0));
}

// `start`: where key k begins (of all waves); every wave's counter of it becomes the place of its first entry
__device__ inline void wave_starts(int *counters, int waves, int pitch, int k, int start)
{
    int at = start;
    for (int w = 0; w < waves; ++w) {
        const int c = counters[w * pitch + k];
        counters[w * pitch + k] = at;
        at += c;
    }
}

// Lists of up to 1024 U places, a bucket a workgroup: every workgroup reads the whole list once and keeps the keys of its own bucket in
// registers, U a lane.  16384 places take 13 us so and 15 over a split list, whose launches are three; 65536 take 96 (every workgroup reads
// half a megabyte) and 21.
template <int U>
__global__ __launch_bounds__(kSortThreads) void embed_short_kernel(SortArgs a)
{
    extern __shared__ int counters[];    // [waves][keys], then the waves' sums
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, me = blockIdx.x;
    int *sums = counters + kSortWaves * a.keys, *mine = counters + wave * a.keys;
    const int lo = wave * (64 * U), keys = (a.rows - me + a.nb - 1) >> a.shift;
    for (int k = threadIdx.x; k < kSortWaves * a.keys; k += kSortThreads) counters[k] = 0;
    __syncthreads();
    uint32_t held[U / 2];                // keys and one, in pairs; 0: another bucket's
    int below = 0;                       // places of the buckets in front of this one
    constexpr int B = U < 16 ? U : 16;
#pragma unroll
    for (int u0 = 0; u0 < U; u0 += B) {
        int t[B];
#pragma unroll
        for (int u = 0; u < B; ++u) t[u] = index_of(a, lo + 64 * (u0 + u) + lane, a.n);
#pragma unroll
        for (int u = 0; u < B; ++u) {
            const int bucket = t[u] & (a.nb - 1);
            below += t[u] >= 0 && bucket < me ? 1 : 0;
            const int key = t[u] >= 0 && bucket == me ? t[u] >> a.shift : -1;
            if (key >= 0) atomicAdd(&mine[key], 1);
            held[(u0 + u) / 2] = u % 2 ? held[(u0 + u) / 2] | (uint32_t)(key + 1) << 16 : (uint32_t)(key + 1);
        }
        __builtin_amdgcn_sched_barrier(0);           // (more loads at once would not fit the registers)
    }
    int base;
    (void)scan_exclusive(below, sums, base);         // (its barrier stands behind the counting too)
    for (int k0 = 0; k0 < keys; k0 += kSortThreads) {
        const int k = k0 + (int)threadIdx.x;
        int n = 0, all;
        if (k < keys)
            for (int w = 0; w < kSortWaves; ++w) n += counters[w * a.keys + k];
        const int start = base + scan_exclusive(n, sums, all);
        base += all;
        if (k < keys) {
            wave_starts(counters, kSortWaves, a.keys, k, start);
            a.run[me + (k << a.shift)] = int2{start, n};
        }
    }
    if (threadIdx.x == 0 && me == (int)gridDim.x - 1) *a.total = base;
    __syncthreads();
    // place the entries in order of the places: few of a round are this bucket's, or many of one key.  (A wave's counters are its own: its
    // reads and writes of them are in order, and `volatile` keeps every one of them.)
    volatile int *next = mine;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int key = (int)(u % 2 ? held[u / 2] >> 16 : held[u / 2] & 0xffffu) - 1;
        uint64_t left = __ballot(key >= 0);
        while (left) {
            const int k = __builtin_amdgcn_readlane(key, __builtin_ctzll(left));
            const uint64_t same = __ballot(key == k);
            const int at = next[k];
            if (key == k) a.sorted[at + lanes_below(same)] = int2{me + (k << a.shift), lo + 64 * u + lane};
            if (lane == 0) next[k] = at + __popcll(same);
            left &= ~same;
        }
    }
}

template <int MODE>
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(SortArgs a)
{
    extern __shared__ int counters[];    // [waves][keys], then the waves' sums
    const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    int *sums = counters + waves * a.keys, *mine = counters + wave * a.keys;
    const int me = blockIdx.x;           // bucket or slice
    // the list: places from .. to - 1, or entries of `split`
    int from, to;
    if constexpr (MODE == kSplitList) {
        from = me * a.slice;
        to = min(a.n, from + a.slice);
    } else {
        from = a.first[me];
        to = a.first[me + 1];
    }
    const int keys = MODE == kSplitList ? a.nb : (a.rows - me + a.nb - 1) >> a.shift;
    const int bits = 32 - __builtin_clz(max(keys - 1, 1));
    for (int k = threadIdx.x; k < waves * a.keys; k += blockDim.x) counters[k] = 0;
    __syncthreads();
    // each wave a part of the list, whole rounds of 64
    const int part = ((max(to - from, 0) + waves - 1) / waves + 63) & ~63;
    const int lo = min(to, from + wave * part), hi = min(to, lo + part);
    auto entry = [&](int i, int &t, int &place) {
        if constexpr (MODE == kBucket) {
            const int2 e = i < hi ? a.split[i] : int2{-1, 0};
            t = e.x;
            place = e.y;
        } else {
            t = index_of(a, i, hi);
            place = i;
        }
    };
    auto key_of = [&](int t) { return t < 0 ? -1 : MODE == kSplitList ? t & (a.nb - 1) : t >> a.shift; };
    // a wave's counters are its own: its lanes' reads and writes of them are in order, and `volatile` keeps every one of them
    volatile int *next = mine;

    for (int i0 = lo; i0 < hi; i0 += 512) {
        int t[8], place;
#pragma unroll
        for (int u = 0; u < 8; ++u) entry(i0 + 64 * u + lane, t[u], place);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if constexpr (MODE == kSplitList) {
                if (t[u] >= 0) atomicAdd(&mine[key_of(t[u])], 1);
            } else {
                // (in a bucket many lanes may have one key, whose additions would wait for each other)
                if (i0 + 64 * u >= hi) break;
                const uint64_t same = same_keys(key_of(t[u]), bits);
                if ((same >> lane) == 1) next[key_of(t[u])] = next[key_of(t[u])] + __popcll(same);
            }
        }
    }
    __syncthreads();
    // where the keys begin, and every wave's part of them
    int base = MODE == kBucket ? from : 0, all;
    for (int k0 = 0; k0 < keys; k0 += blockDim.x) {
        const int k = k0 + (int)threadIdx.x;
        int n = 0, before = 0;           // of the whole workgroup; split lists: of all slices, and of those in front of this one
        if (k < keys) {
            if constexpr (MODE == kSplitList) {
                int h[kSlices];
#pragma unroll
                for (int s = 0; s < kSlices; ++s) h[s] = a.hist[(size_t)s * a.nb + k];
#pragma unroll
                for (int s = 0; s < kSlices; ++s) {
                    n += h[s];
                    before += s < me ? h[s] : 0;
                }
            } else {
                for (int w = 0; w < waves; ++w) n += counters[w * a.keys + k];
            }
        }
        const int start = base + scan_exclusive(n, sums, all);
        base += all;
        if (k < keys) {
            wave_starts(counters, waves, a.keys, k, start + before);
            if constexpr (MODE == kSplitList) {
                if (me == 0) a.first[k] = start;
                if (me == 0 && a.rows <= a.nb && k < a.rows) a.run[k] = int2{start, n};
            } else {
                a.run[me + (k << a.shift)] = int2{start, n};
            }
        }
    }
    if (MODE == kSplitList && threadIdx.x == 0 && me == 0) *a.total = a.first[a.nb] = base;
    __syncthreads();
    // place the entries in order of the list
    int2 *out = MODE == kSplitList && a.rows > a.nb ? a.split : a.sorted;
    for (int i0 = lo; i0 < hi; i0 += 512) {
        int t[8], place[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) entry(i0 + 64 * u + lane, t[u], place[u]);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (i0 + 64 * u >= hi) break;
            const int key = key_of(t[u]);
            const uint64_t same = same_keys(key, bits);
            if (key >= 0) {
                const int at = next[key];
                out[at + lanes_below(same)] = int2{t[u], place[u]};
                if ((same >> lane) == 1) next[key] = at + __popcll(same);       // the last of them
            }
        }
    }
}

// ---- sums ----------------------------------------------------------------------------------------------------------
struct SumArgs {
    const void *dy;
    void *dw;
    const int2 *sorted, *run;
    const int *total;
    float *part;          // [chunks][2][pitch]: the end of a run from earlier chunks (or one that fills the chunk), a run that goes on
    int C, pitch, chunk;  // chunk: places of a chunk, a multiple of 8
    int n;                // places in all (of which *total count)
    int rows;
    int blocks, tiles;    // workgroups of the sums along the places and along the columns; those behind them write the rows of zeros
    float scale;
};
constexpr int kZeroVectors = 4 * kThreads;      // of a workgroup that writes zeros

template <int DT, int WT> __device__ inline void store_row(const SumArgs &a, int row, const Part &p, const float (&s)[NormElem<DT>::V])
{
    constexpr int V = NormElem<DT>::V, VW = NormElem<WT>::V;
    typedef typename NormElem<WT>::t elem_t;
    elem_t *w = static_cast<elem_t *>(a.dw) + (size_t)row * a.C;
#pragma unroll
    for (int j = 0; j < V; j += VW) {
        float t[VW];
#pragma unroll
        for (int i = 0; i < VW; ++i) t[i] = s[j + i] * a.scale;
        const Part q{p.at + j, 0, min(VW, p.hi - j)};
        if (q.hi > 0) store_part<WT>(w, pack<WT>(t), q);
    }
}

// G lanes lie along the columns, a group takes a chunk
template <int DT, int WT, int G>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(SumArgs a)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, RP = kThreads / G, U = 8;
    const int nv = (a.C + V - 1) / V, exact = a.C < V;
    if ((int)blockIdx.x >= a.blocks * a.tiles) {
        float zero[V];
#pragma unroll
        for (int i = 0; i < V; ++i) zero[i] = 0.f;
        const long long first = (long long)((int)blockIdx.x - a.blocks * a.tiles) * kZeroVectors + threadIdx.x, all = (long long)a.rows * nv;
        for (long long v0 = first; v0 < all; v0 += (long long)((int)gridDim.x - a.blocks * a.tiles) * kZeroVectors)
#pragma unroll
            for (int u = 0; u < kZeroVectors / kThreads; ++u) {
                const long long q = v0 + u * kThreads;
                const int row = (int)(all < (1LL << 31) ? (uint32_t)q / (uint32_t)nv : q / nv);
                if (row < a.rows && a.run[row].y == 0) store_row<DT, WT>(a, row, part_of<V>((int)(q - (long long)row * nv), a.C, exact), zero);
            }
        return;
    }
    const int tile = (int)blockIdx.x % a.tiles, chunk = (int)blockIdx.x / a.tiles * RP + threadIdx.x / G, v = tile * G + threadIdx.x % G;
    const long long from = (long long)chunk * a.chunk;
    if (from >= a.n || v >= nv) return;
    // (entries past the total are not written, and count for nothing)
    const int lo = (int)from, total = *a.total, hi = (int)min((long long)total, from + a.chunk);
    int2 e[U], before = a.sorted[max(lo - 1, 0)];
#pragma unroll
    for (int u = 0; u < U; ++u) e[u] = a.sorted[min(lo + u, a.n - 1)];
    if (lo >= total) return;
    const Part p = part_of<V>(v, a.C, exact);
    const elem_t *DY = static_cast<const elem_t *>(a.dy);
    float s[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = 0.f;
    int cur = e[0].x;
    bool open = lo > 0 && before.x == cur;                   // the run began in an earlier chunk
    auto leave = [&](bool goes_on) {
        if (!open && !goes_on) {
            store_row<DT, WT>(a, cur, p, s);
        } else {
            float *q = a.part + ((size_t)chunk * 2 + (open ? 0 : 1)) * a.pitch;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < p.hi) q[p.at + i] = s[i];
        }
    };
    for (int e0 = lo; e0 < hi; e0 += U) {
        uint4 raw[U];
        int2 ahead[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = e0 + u < hi ? load_part<DT>(DY + (size_t)e[u].y * a.C, p) : uint4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < U; ++u) ahead[u] = a.sorted[min(e0 + U + u, a.n - 1)];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (e0 + u >= hi) break;
            if (e[u].x != cur) {
                leave(false);
                cur = e[u].x;
                open = false;
#pragma unroll
                for (int i = 0; i < V; ++i) s[i] = 0.f;
            }
            float t[V];
            unpack<DT>(raw[u], t);
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] += t[i];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) e[u] = ahead[u];
    }
    leave(hi < total && a.sorted[hi].x == cur);
}

// Small gradients in one launch: a bucket a workgroup as in embed_short_kernel, whose places stay in LDS and are added up right there.  Runs
// of up to kSmallRun places are a wave's, longer ones are shared by the waves and joined in order.
// 1999 places of 5003 x 300 fp16: 8.3 us (14.4 in three launches).
constexpr int kSmallList = 4 * kSortThreads, kSmallKeys = 256, kSmallRun = 16;
template <int DT, int WT>
__global__ __launch_bounds__(kSortThreads) void embed_small_kernel(SortArgs a, SumArgs m)
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V, U = kSmallList / kSortThreads;
    extern __shared__ int counters[];    // [waves][keys], then the waves' sums
    __shared__ uint16_t order[kSmallList], few[kSmallKeys], many[kSmallKeys];
    __shared__ int2 runs[kSmallKeys];
    __shared__ int nfew, nmany;
    __shared__ float part[kSortWaves][64 * V];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, me = blockIdx.x;
    int *sums = counters + kSortWaves * a.keys, *mine = counters + wave * a.keys;
    const int lo = wave * (64 * U), keys = (a.rows - me + a.nb - 1) >> a.shift;
    for (int k = threadIdx.x; k < kSortWaves * a.keys; k += kSortThreads) counters[k] = 0;
    if (threadIdx.x == 0) nfew = nmany = 0;
    __syncthreads();
    int key[U];
#pragma unroll
    for (int u = 0; u < U; ++u) key[u] = index_of(a, lo + 64 * u + lane, a.n);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        key[u] = key[u] >= 0 && (key[u] & (a.nb - 1)) == me ? key[u] >> a.shift : -1;
        if (key[u] >= 0) atomicAdd(&mine[key[u]], 1);
    }
    __syncthreads();
    const int k = threadIdx.x;
    int n = 0, all;
    if (k < keys)
        for (int w = 0; w < kSortWaves; ++w) n += counters[w * a.keys + k];
    const int start = scan_exclusive(n, sums, all);
    if (k < keys) {
        wave_starts(counters, kSortWaves, a.keys, k, start);
        runs[k] = int2{start, n};
        // (in any order: every row is added up by itself)
        if (n > kSmallRun) many[atomicAdd(&nmany, 1)] = (uint16_t)k;
        else if (n > 0) few[atomicAdd(&nfew, 1)] = (uint16_t)k;
    }
    __syncthreads();
    volatile int *next = mine;           // (as in embed_short_kernel)
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint64_t left = __ballot(key[u] >= 0);
        while (left) {
            const int q = __builtin_amdgcn_readlane(key[u], __builtin_ctzll(left));
            const uint64_t same = __ballot(key[u] == q);
            const int at = next[q];
            if (key[u] == q) order[at + lanes_below(same)] = (uint16_t)(lo + 64 * u + lane);
            if (lane == 0) next[q] = at + __popcll(same);
            left &= ~same;
        }
    }
    __syncthreads();
    const int nv = (m.C + V - 1) / V, exact = m.C < V, tiles = (nv + 63) / 64;
    const elem_t *DY = static_cast<const elem_t *>(m.dy);
    // the places first .. first + count - 1 of the bucket, this lane's vector
    auto add = [&](int first, int count, const Part &p, float (&s)[V]) {
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = 0.f;
        for (int e0 = 0; e0 < count; e0 += 8) {
            uint4 raw[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) raw[u] = e0 + u < count ? load_part<DT>(DY + (size_t)order[first + e0 + u] * m.C, p) : uint4{0, 0, 0, 0};
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (e0 + u >= count) break;
                float t[V];
                unpack<DT>(raw[u], t);
#pragma unroll
                for (int i = 0; i < V; ++i) s[i] += t[i];
            }
        }
    };
    for (int q = wave; q < nfew * tiles; q += kSortWaves) {
        const int f = few[q / tiles], v = q % tiles * 64 + lane;
        if (v >= nv) continue;
        const Part p = part_of<V>(v, m.C, exact);
        float s[V];
        add(runs[f].x, runs[f].y, p, s);
        store_row<DT, WT>(m, me + (f << a.shift), p, s);
    }
    for (int q = 0; q < nmany * tiles; ++q) {        // (the same count for all threads)
        const int f = many[q / tiles], v = q % tiles * 64 + lane;
        const Part p = part_of<V>(v, m.C, exact);
        const int2 r = runs[f];
        const int share = (r.y + kSortWaves - 1) / kSortWaves, first = min(r.y, wave * share), count = min(r.y - first, share);
        float s[V];
        if (v < nv) {
            add(r.x + first, count, p, s);
#pragma unroll
            for (int i = 0; i < V; ++i) part[wave][lane * V + i] = s[i];
        }
        __syncthreads();
        if (wave == 0 && v < nv) {
            for (int w = 1; w < kSortWaves; ++w)
#pragma unroll
                for (int i = 0; i < V; ++i) s[i] += part[w][lane * V + i];
            store_row<DT, WT>(m, me + (f << a.shift), p, s);
        }
        __syncthreads();
    }
    // rows that no place names
    float zero[V];
#pragma unroll
    for (int i = 0; i < V; ++i) zero[i] = 0.f;
    const long long vectors = (long long)keys * nv;
    for (long long q = threadIdx.x; q < vectors; q += kSortThreads) {
        const int f = (int)(vectors < (1LL << 31) ? (uint32_t)q / (uint32_t)nv : q / nv);
        if (runs[f].y == 0) store_row<DT, WT>(m, me + (f << a.shift), part_of<V>((int)(q - (long long)f * nv), m.C, exact), zero);
    }
}

// the runs that cross chunks, a workgroup each: 64 lanes along 256 columns, the waves share the chunks
constexpr int kJoinWaves = 4;
template <int WT>
__global__ __launch_bounds__(kJoinWaves * 64) void embed_join_kernel(SumArgs a)
{
    __shared__ float4 red[kJoinWaves][64];
    const int chunk = blockIdx.x;
    const long long end = ((long long)chunk + 1) * a.chunk;      // (below n: the last chunk has no workgroup)
    const int total = *a.total, t = a.sorted[end - 1].x, behind = a.sorted[end].x;
    if (end >= total || behind != t) return;
    const int2 run = a.run[t];
    if (run.x < (long long)chunk * a.chunk) return;          // it began in an earlier chunk, whose workgroup joins it
    const int n = (run.x + run.y - 1) / a.chunk - chunk + 1; // chunks
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (blockIdx.y * 64 + lane) * 4;
    const float *part = a.part + (size_t)chunk * 2 * a.pitch;
    float4 s{0.f, 0.f, 0.f, 0.f};
    if (c < a.C) {
#pragma unroll 16
        for (int k = wave; k < n; k += kJoinWaves) {
            const float4 q = *reinterpret_cast<const float4 *>(part + ((size_t)k * 2 + (k == 0 ? 1 : 0)) * a.pitch + c);
            s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
        }
    }
    red[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= a.C) return;
    for (int w = 1; w < min(n, kJoinWaves); ++w) {
        const float4 q = red[w][lane];
        s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
    }
    const float v[4] = {s.x, s.y, s.z, s.w};
    typename NormElem<WT>::t *w = static_cast<typename NormElem<WT>::t *>(a.dw) + (size_t)t * a.C;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (c + i < a.C) w[c + i] = norm_round<WT>(v[i] * a.scale);
}

__global__ __launch_bounds__(kThreads) void embed_zero_kernel(uint8_t *p, size_t n)
{
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (size_t)gridDim.x * kThreads) p[i] = 0;
}

// ---- launches ------------------------------------------------------------------------------------------------------
constexpr int kShortList = 16 * kSortThreads;

struct EmbedPlan {
    int nb, shift, keys;
    bool small;                         // one launch sorts
    bool once;                          // one launch does everything
    int chunk, chunks, pitch, G, tiles;
    size_t sorted, split, run, hist, first, total, part, bytes;
};
int column_lanes(int nv)
{
    for (int G : {8, 16, 32})
        if (nv <= G) return G;
    return 64;
}
EmbedPlan embed_plan(const xconv_embed_desc *d)
{
    EmbedPlan p{};
    p.shift = 8;
    while ((d->rows + (1LL << p.shift) - 1) >> p.shift > kSortKeys) ++p.shift;
    p.nb = 1 << p.shift;
    p.keys = (int)((d->rows + p.nb - 1) >> p.shift);
    p.small = d->n <= kShortList && p.shift == 8;
    // a workgroup adds up what its bucket has: of lists whose places might all name one row, no more than it reads in a few microseconds
    const long long bytes = d->n * d->C * (d->dtype == XCONV_F32 ? 4 : 2);
    p.once = p.small && d->n <= kSmallList && p.keys <= kSmallKeys && bytes <= (1 << 21) && bytes / std::min<long long>(p.nb, d->rows) <= (1 << 17);
    const int V = d->dtype == XCONV_F32 ? 4 : 8, nv = ceil_div(d->C, V);
    p.G = column_lanes(nv);
    p.tiles = ceil_div(nv, p.G);
    // a few thousand waves where there is work for them; chunks long enough that few runs cross them and few partial sums make up a long run
    p.chunk = 8;
    while (p.chunk < 256 && (d->n / p.chunk > 8192 || d->n / p.chunk * p.tiles * p.G / 64 > 2048)) p.chunk *= 2;
    p.chunks = (int)((d->n + p.chunk - 1) / p.chunk);
    p.pitch = round_up(d->C, 4);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t a = at;
        at += (bytes + 255) / 256 * 256;
        return a;
    };
    p.sorted = take((size_t)d->n * 8);
    p.run = take((size_t)d->rows * 8);
    p.total = take(4);
    if (!p.small) {
        p.split = take((size_t)d->n * 8);
        p.hist = take((size_t)kSlices * p.nb * 4);
        p.first = take(((size_t)p.nb + 1) * 4);
    }
    p.part = take((size_t)p.chunks * 2 * p.pitch * 4);
    p.bytes = at;
    return p;
}

template <int DT, int WT> hipError_t go_sum(const SumArgs &a, const SortArgs &sort, const EmbedPlan &p, hipStream_t st)
{
    SumArgs s = a;
    if (p.once) {
        const dim3 grid((unsigned)std::min<long long>(p.nb, a.rows));
        hipLaunchKernelGGL((embed_small_kernel<DT, WT>), grid, dim3(kSortThreads), (size_t)(kSortWaves * p.keys + kSortWaves) * 4, st, sort, s);
        return hipGetLastError();
    }
    const int rp = kThreads / p.G;
    s.blocks = ceil_div(p.chunks, rp);
    constexpr int V = NormElem<DT>::V;
    const long long zeros = std::min<long long>(((long long)a.rows * ceil_div(a.C, V) + kZeroVectors - 1) / kZeroVectors, 1 << 20);
    s.tiles = p.tiles;
    const dim3 grid((unsigned)((long long)s.blocks * s.tiles + zeros)), block(kThreads);
    switch (p.G) {
    case 8: hipLaunchKernelGGL((embed_sum_kernel<DT, WT, 8>), grid, block, 0, st, s); break;
    case 16: hipLaunchKernelGGL((embed_sum_kernel<DT, WT, 16>), grid, block, 0, st, s); break;
    case 32: hipLaunchKernelGGL((embed_sum_kernel<DT, WT, 32>), grid, block, 0, st, s); break;
    default: hipLaunchKernelGGL((embed_sum_kernel<DT, WT, 64>), grid, block, 0, st, s); break;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.chunks < 2) return e;
    hipLaunchKernelGGL(embed_join_kernel<WT>, dim3((unsigned)(p.chunks - 1), (unsigned)ceil_div(a.C, 256)), dim3(kJoinWaves * 64), 0, st, s);
    return hipGetLastError();
}

template <int DT, int G> void go_lookup(const LookupArgs &a, int tiles, hipStream_t st)
{
    // four places a group where that leaves enough workgroups
    constexpr int RP = kThreads / G;
    const long long one = (a.n + RP - 1) / RP, four = (a.n + 4 * RP - 1) / (4 * RP);
    if (four * tiles >= 2048) hipLaunchKernelGGL((embed_lookup_kernel<DT, G, 4>), dim3((unsigned)std::min<long long>(four, 1 << 20), (unsigned)tiles), dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((embed_lookup_kernel<DT, G, 1>), dim3((unsigned)std::min<long long>(one, 1 << 20), (unsigned)tiles), dim3(kThreads), 0, st, a);
}
template <int DT> hipError_t launch_lookup_dt(const LookupArgs &a, hipStream_t st)
{
    constexpr int V = NormElem<DT>::V;
    const int nv = ceil_div(a.C, V);
    if (nv <= 8) go_lookup<DT, 8>(a, 1, st);
    else if (nv <= 16) go_lookup<DT, 16>(a, 1, st);
    else if (nv <= 32) go_lookup<DT, 32>(a, 1, st);
    else if (nv <= 64) go_lookup<DT, 64>(a, 1, st);
    else go_lookup<DT, 256>(a, std::min(ceil_div(nv, 256), 64), st);
    return hipGetLastError();
}

}  // namespace

size_t embed_ws_bytes(const xconv_embed_desc *d) { return embed_plan(d).bytes; }

hipError_t launch_embed_fwd(const xconv_embed_desc *d, const void *idx, const void *W, void *Y, hipStream_t st)
{
    const LookupArgs a{idx, W, Y, d->n, d->rows, d->C, d->index64, d->scale};
    if (d->dtype == XCONV_F32) return launch_lookup_dt<XCONV_F32>(a, st);
    return d->dtype == XCONV_BF16 ? launch_lookup_dt<XCONV_BF16>(a, st) : launch_lookup_dt<XCONV_F16>(a, st);
}

hipError_t launch_embed_bwd(const xconv_embed_desc *d, const void *idx, const void *dY, void *dW, int dw_dtype, void *ws, hipStream_t st)
{
    if (d->n == 0) {
        const size_t bytes = (size_t)d->rows * d->C * (dw_dtype == XCONV_F32 ? 4 : 2);
        hipLaunchKernelGGL(embed_zero_kernel, dim3((unsigned)std::min<size_t>((bytes + kThreads - 1) / kThreads, 2048)), dim3(kThreads), 0, st, static_cast<uint8_t *>(dW), bytes);
        return hipGetLastError();
    }
    const EmbedPlan p = embed_plan(d);
    char *base = static_cast<char *>(ws);
    SortArgs s{};
    s.idx = idx;
    s.wide = d->index64;
    s.n = (int)d->n;
    s.rows = (int)d->rows;
    s.pad = d->padding_idx;
    s.nb = p.nb;
    s.shift = p.shift;
    s.keys = p.keys;
    s.sorted = reinterpret_cast<int2 *>(base + p.sorted);
    s.run = reinterpret_cast<int2 *>(base + p.run);
    s.total = reinterpret_cast<int *>(base + p.total);
    auto lds = [](int waves, int keys) { return (size_t)(waves * keys + waves) * 4; };
    if (p.once) {
        // (everything below)
    } else if (p.small) {
        const dim3 grid((unsigned)std::min<long long>(p.nb, d->rows)), block(kSortThreads);
        const size_t l = lds(kSortWaves, p.keys);
        if (d->n <= 4 * kSortThreads) hipLaunchKernelGGL(embed_short_kernel<4>, grid, block, l, st, s);
        else hipLaunchKernelGGL(embed_short_kernel<16>, grid, block, l, st, s);
    } else {
        s.split = reinterpret_cast<int2 *>(base + p.split);
        s.hist = reinterpret_cast<int *>(base + p.hist);
        s.first = reinterpret_cast<int *>(base + p.first);
        s.slice = (int)((d->n + kSlices - 1) / kSlices);
        hipLaunchKernelGGL(embed_count_kernel, dim3(kSlices), dim3(kSortThreads), (size_t)p.nb * 4, st, s);
        SortArgs t = s;
        t.keys = p.nb;
        // as many waves as have room for counters of all buckets
        const int waves = std::max(1, std::min(kSortWaves, 15 * 1024 / p.nb));
        hipLaunchKernelGGL(embed_sort_kernel<kSplitList>, dim3(kSlices), dim3(waves * 64), lds(waves, p.nb), st, t);
        if (d->rows > p.nb) hipLaunchKernelGGL(embed_sort_kernel<kBucket>, dim3((unsigned)p.nb), dim3(kSortThreads), lds(kSortWaves, p.keys), st, s);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    SumArgs a{};
    a.dy = dY;
    a.dw = dW;
    a.sorted = s.sorted;
    a.run = s.run;
    a.total = s.total;
    a.part = reinterpret_cast<float *>(base + p.part);
    a.n = (int)d->n;
    a.C = d->C;
    a.pitch = p.pitch;
    a.chunk = p.chunk;
    a.rows = (int)d->rows;
    a.scale = d->scale;
    if (d->dtype == XCONV_F32) return go_sum<XCONV_F32, XCONV_F32>(a, s, p, st);
    const bool w32 = dw_dtype == XCONV_F32;
    if (d->dtype == XCONV_BF16) return w32 ? go_sum<XCONV_BF16, XCONV_F32>(a, s, p, st) : go_sum<XCONV_BF16, XCONV_BF16>(a, s, p, st);
    return w32 ? go_sum<XCONV_F16, XCONV_F32>(a, s, p, st) : go_sum<XCONV_F16, XCONV_F16>(a, s, p, st);
}

}  // namespace xc
