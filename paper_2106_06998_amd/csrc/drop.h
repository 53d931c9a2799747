// Masks of dropout, drawn where they are applied and never stored: value e of a tensor in memory order takes bits 16 (e%4) .. +15 of
// word e/4 of the SplitMix64 stream (common.h) of (seed + *step) xor kDropStream, and is dropped where they are below q16; the others are
// multiplied by 65536 / (65536 - q16).  A word serves four values: about eleven instructions each, six of them quarter-rate products.
#pragma once
#include "common.h"

namespace xc {

constexpr uint64_t kDropStream = 0x3C6EF372FE94F82Bull;

struct DropArgs {
    uint64_t seed;
    const long long *step;   // on the device, or null for 0
    uint32_t q16;            // of 65536 values so many are dropped; 0: none are, and no words are drawn
    float scale;             // 65536 / (65536 - q16), 0 where all are dropped
};

inline DropArgs drop_args(const xconv_drop *d)
{
    if (!d || d->drop_q16 == 0) return DropArgs{0, nullptr, 0, 1.f};
    return DropArgs{d->seed, reinterpret_cast<const long long *>(d->step_dev), (uint32_t)d->drop_q16, d->drop_q16 == 65536 ? 0.f : (float)(65536.0 / (65536 - d->drop_q16))};
}

__host__ __device__ inline uint64_t drop_key(uint64_t seed, uint64_t step)
{
    return mix_fin(((seed + step) ^ kDropStream) + 0x9E3779B97F4A7C15ull);
}
__device__ inline uint64_t drop_key(const DropArgs &d) { return drop_key(d.seed, d.step ? (uint64_t)*d.step : 0); }

// x <- what dropout makes of the V values from place e on.  fours: e is a multiple of 4 in every call of the launch
template <int V> __device__ inline void drop_values(const DropArgs &d, uint64_t key, uint64_t e, bool fours, float (&x)[V])
{
    uint64_t w[V / 4];
    if (fours) {
#pragma unroll
        for (int j = 0; j < V / 4; ++j) w[j] = stream_word(key, (e >> 2) + j);
    } else {
        uint64_t u[V / 4 + 1];
#pragma unroll
        for (int j = 0; j <= V / 4; ++j) u[j] = stream_word(key, (e >> 2) + j);
        const int s = 16 * (int)(e & 3);
#pragma unroll
        for (int j = 0; j < V / 4; ++j) w[j] = (u[j] >> s) | ((u[j + 1] << 1) << (63 - s));
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t half = (uint32_t)(w[i / 4] >> (32 * (i / 2 % 2)));
        const uint32_t field = i % 2 ? half >> 16 : half & 0xffffu;
        x[i] = field >= d.q16 ? x[i] * d.scale : 0.f;
    }
}

}  // namespace xc
