// What the kernels share that take a head's elements eight to a lane: sums over the lanes of a head, the header's types.
#pragma once

#include "../../include/positnn_generate.h"
#include "lm_codec.h"

namespace pnn {

// Of L lanes in a row (a power of two up to 32), in each of them; all of the L call.  Within 16 lanes through the vector unit's own lane
// shifts: once the lanes of a block are alike, a mirrored block is its neighbour's.
template <int L, class F>
__device__ __forceinline__ uint32_t group_fold(uint32_t v, F f) {
    static_assert(L <= 32, "");
    if (L >= 2) v = f(v, lane_shift<0xB1, 0xF>(v, 0u));
    if (L >= 4) v = f(v, lane_shift<0x4E, 0xF>(v, 0u));
    if (L >= 8) v = f(v, lane_shift<0x141, 0xF>(v, 0u));
    if (L >= 16) v = f(v, lane_shift<0x140, 0xF>(v, 0u));
    if (L >= 32) v = f(v, (uint32_t)__shfl_xor((int)v, 16, 64));
    return v;
}
template <int L>
__device__ __forceinline__ float group_sum(float v) {
    return f32_of_bits(group_fold<L>(bits_of_f32(v), [](uint32_t x, uint32_t y) { return bits_of_f32(f32_of_bits(x) + f32_of_bits(y)); }));
}
template <int L>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
    return group_fold<L>(v, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
}
template <int L>
__device__ __forceinline__ double group_sum(double v) {
    static_assert(L <= 32, "");
    auto step = [&](auto shift) {
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        v += __builtin_bit_cast(double, (uint64_t)shift((uint32_t)(b >> 32)) << 32 | shift((uint32_t)b));
    };
    if (L >= 2) step([](uint32_t x) { return lane_shift<0xB1, 0xF>(x, 0u); });
    if (L >= 4) step([](uint32_t x) { return lane_shift<0x4E, 0xF>(x, 0u); });
    if (L >= 8) step([](uint32_t x) { return lane_shift<0x141, 0xF>(x, 0u); });
    if (L >= 16) step([](uint32_t x) { return lane_shift<0x140, 0xF>(x, 0u); });
    if (L >= 32) step([](uint32_t x) { return (uint32_t)__shfl_xor((int)x, 16, 64); });
    return v;
}

// v to binary32 in such a way that a further rounding to fewer bits is that of v: toward zero, the last bit set where anything was cut off
// (NaN and infinities stay; beyond binary32's range its largest number)
__device__ __forceinline__ float f32_to_odd(double v) {
    const float f = (float)v;
    const uint32_t b = bits_of_f32(f);
    const double back = (double)f;
    if (back == v || v != v) return f;
    const bool over = (back < 0.0 ? -back : back) > (v < 0.0 ? -v : v);
    return f32_of_bits((over ? b - 1u : b) | 1u);
}

}  // namespace pnn
