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
// The same of eight, where it matters: the nearest number of binary32 lies on the same side of every border of two results as v does, unless it is that border, whose last bits (`zeros`) are
// zero.  Borders of 8-bit posits, bfloat16 and 4 bits have at most 10 significant bits, those of 16-bit posits 14.
constexpr uint32_t ZEROS_8 = 0x3FFFu, ZEROS_16 = 0x3FFu;
__device__ __forceinline__ void f32_for_rounding(float (&v)[8], const double (&x)[8], uint32_t zeros) {
    uint32_t least = ~0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] = (float)x[e];
        const uint32_t low = bits_of_f32(v[e]) & zeros;
        least = low < least ? low : least;
    }
    if (least == 0u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = f32_to_odd(x[e]);
    }
}

// 1 / sqrt(x) in binary64 for positive x: the instruction's 24 bits or so, doubled twice; 0 and infinity where it gives infinity and 0
__device__ __forceinline__ double rsqrt_wide(double x) {
    double y = __builtin_amdgcn_rsq(x);
    if (!(x > 1e-290 && x < 1e290)) return 1.0 / sqrt(x);
#pragma unroll
    for (int i = 0; i < 2; ++i) y = fma(y * 0.5, fma(-x * y, y, 1.0), y);
    return y;
}

// A lane's elements: 0 .. 3 the firsts of its four pairs and 4 .. 7 the seconds, or, of neighbours, as they lie.  WHOLE: both runs of four are inside a head and on one side of R / 2, of
// every lane (heads_whole); else each element is looked at by itself.
template <bool NEIGHBOURS, bool WHOLE>
struct HeadLane {
    int lane, D, R, run0, run1;
    bool in;  // WHOLE: the lane has elements
    // element of the head, or -1
    __device__ __forceinline__ int first(int e) const {
        const int half = R / 2, rest = (D - R) / 2, p = 4 * lane + (NEIGHBOURS ? e / 2 : e & 3), second = NEIGHBOURS ? e & 1 : e >> 2;
        if (WHOLE) return in ? (e < 4 ? run0 : run1) + (e & 3) : -1;
        if (p >= D / 2) return -1;
        return NEIGHBOURS ? 2 * p + second : (p < half ? p + second * half : R + (p - half) + second * rest);
    }
    __device__ __forceinline__ HeadLane(int lane, int D, int R) : lane(lane), D(D), R(R) {
        const int half = R / 2, p = 4 * lane;
        in = p < D / 2;
        run0 = NEIGHBOURS ? 2 * p : (p < half ? p : R + (p - half));
        run1 = NEIGHBOURS ? 2 * p + 4 : (p < half ? p + half : R + (p - half) + (D - R) / 2);
    }
};
inline bool heads_whole(int64_t D, int64_t R, bool neighbours) { return D % 8 == 0 && (neighbours || R % 8 == 0); }

template <bool NEIGHBOURS, bool WHOLE>
__device__ __forceinline__ void heads_load(Raw8& r, const HeadLane<NEIGHBOURS, WHOLE>& l, const void* p, int64_t at, int kind) {
    r.w = (words8)(0u);
    if (WHOLE) {
        if (!l.in) return;
        if (NEIGHBOURS) {
            load8(r, p, at + l.run0, kind, 8);
        } else if (kind == KIND_POSIT_U8) {
            uint32_t b[2];
            __builtin_memcpy(&b[0], (const uint8_t*)p + at + l.run0, 4);
            __builtin_memcpy(&b[1], (const uint8_t*)p + at + l.run1, 4);
            r.w[0] = b[0];
            r.w[1] = b[1];
        } else if (kind == KIND_F32) {
            r.w.lo = *(const words4_any*)((const uint32_t*)p + at + l.run0);
            r.w.hi = *(const words4_any*)((const uint32_t*)p + at + l.run1);
        } else {
            r.w.lo.lo = *(const words2_any*)((const uint16_t*)p + at + l.run0);
            r.w.lo.hi = *(const words2_any*)((const uint16_t*)p + at + l.run1);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (l.first(e) < 0) continue;
        const int64_t i = at + l.first(e);
        if (kind == KIND_POSIT_U8) r.w[e / 4] |= (uint32_t)((const uint8_t*)p)[i] << (8 * (e & 3));
        else if (kind == KIND_F32) r.w[e] = ((const uint32_t*)p)[i];
        else r.w[e / 2] |= (uint32_t)((const uint16_t*)p)[i] << (16 * (e & 1));
    }
}

template <bool NEIGHBOURS, bool WHOLE>
__device__ __forceinline__ void heads_store(const Raw8& r, const HeadLane<NEIGHBOURS, WHOLE>& l, void* p, int64_t at, int kind) {
    if (WHOLE) {
        if (!l.in) return;
        if (NEIGHBOURS) {
            store8(p, at + l.run0, r, kind, 8);
        } else if (kind == KIND_POSIT_U8) {
            const uint32_t b[2] = {r.w[0], r.w[1]};
            __builtin_memcpy((uint8_t*)p + at + l.run0, &b[0], 4);
            __builtin_memcpy((uint8_t*)p + at + l.run1, &b[1], 4);
        } else if (kind == KIND_F32) {
            *(words4_any*)((uint32_t*)p + at + l.run0) = r.w.lo;
            *(words4_any*)((uint32_t*)p + at + l.run1) = r.w.hi;
        } else {
            *(words2_any*)((uint16_t*)p + at + l.run0) = r.w.lo.lo;
            *(words2_any*)((uint16_t*)p + at + l.run1) = r.w.lo.hi;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (l.first(e) < 0) continue;
        const int64_t i = at + l.first(e);
        if (kind == KIND_POSIT_U8) ((uint8_t*)p)[i] = (uint8_t)(r.w[e / 4] >> (8 * (e & 3)));
        else if (kind == KIND_F32) ((uint32_t*)p)[i] = r.w[e];
        else ((uint16_t*)p)[i] = (uint16_t)(r.w[e / 2] >> (16 * (e & 1)));
    }
}

// The lane's first n pairs by their angles, the others as they are (an infinity there would make a NaN of its partner); BACK: by the negatives.  A lane of WHOLE halves has all of its
// pairs before R or none.
template <bool NEIGHBOURS, bool WHOLE, bool BACK, class T, class T2>
__device__ __forceinline__ void heads_turn(T (&v)[8], const T2 (&cs)[4], int n) {
    constexpr int step = NEIGHBOURS ? 2 : 1, gap = NEIGHBOURS ? 1 : 4;
    auto turn = [&](auto all) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = step * i, y = x + gap;
            const T s = BACK ? -cs[i].y : cs[i].y, a = v[x], b = v[y];
            const T ta = __builtin_elementwise_fma(a, cs[i].x, -(b * s)), tb = __builtin_elementwise_fma(b, cs[i].x, a * s);
            v[x] = all() || i < n ? ta : a;
            v[y] = all() || i < n ? tb : b;
        }
    };
    if (n >= 4) turn([] { return true; });
    else if ((!WHOLE || NEIGHBOURS) && n > 0) turn([] { return false; });
}

// Values of 8-bit posits by look-up: 16 copies of each in LDS, so that the lanes of a wave meet few conflicts (three instructions an element where decoding takes 13)
constexpr int HEADS_COPIES = 16;
__device__ __forceinline__ void heads_table(uint32_t* table, ElemFmt f) {
    const uint32_t v = bits_of_f32(posit_value(threadIdx.x, f));
#pragma unroll
    for (int c = 0; c < HEADS_COPIES / 4; ++c) ((uint4*)table)[threadIdx.x * (HEADS_COPIES / 4) + c] = make_uint4(v, v, v, v);
}
__device__ __forceinline__ void heads_look_up(float (&v)[8], const Raw8& r, const uint32_t* table) {
    const uint32_t* const mine = table + (threadIdx.x & (HEADS_COPIES - 1));
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = f32_of_bits(mine[((r.w[e / 4] >> (8 * (e & 3))) & 0xFFu) * HEADS_COPIES]);
}
// 1 / sqrt(x) to a unit in the last place
__device__ __forceinline__ float rsqrt_near(float x) { return x > 1e-30f ? __builtin_amdgcn_rsqf(x) : 1.f / sqrtf(x); }

template <bool NEIGHBOURS, bool WHOLE>
__device__ __forceinline__ void heads_weights(float (&w)[8], const HeadLane<NEIGHBOURS, WHOLE>& l, const void* p, int kind, ElemFmt f) {
    Raw8 raw;
    heads_load(raw, l, p, 0, kind);
    values8(w, raw, kind, f);
}

// The group's heads of a block: one after the other over rows and heads, without divisions
struct HeadItem {
    int r, h, dr, dh, heads;
    __device__ __forceinline__ HeadItem(int group, int groups, int n) : heads(n) {
        r = group / n;
        h = group - r * n;
        dr = groups / n;
        dh = groups - dr * n;
    }
    __device__ __forceinline__ void next() {
        r += dr;
        h += dh;
        if (h >= heads) {
            h -= heads;
            ++r;
        }
    }
};

}  // namespace pnn
