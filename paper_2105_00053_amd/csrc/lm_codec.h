// Elements of the language-model operators: posits of at most 16 bits, bfloat16 and binary32, all read as binary32 (exactly) and
// rounded once when stored.  A posit's format is known at run time (n and es are wave-uniform); what is a template parameter is how an
// element lies in memory.
#pragma once

#include "api_common.h"
#include "../../include/positnn_lm.h"
#include "posit_core.h"

namespace pnn {

enum ElemKind { KIND_POSIT_U8 = 0, KIND_POSIT_U16 = 1, KIND_BF16 = 2, KIND_F32 = 3 };

// The part of a format that a kernel needs beside its kind.
struct ElemFmt {
    int n, es;
};

inline bool is_element(int f) { return (is_posit(f) && f != PNN_POSIT32_2) || f == PNN_F32 || f == PNN_BF16; }
// PNN_OK for an element format, else what an entry point returns for it
inline int element_status(int f) { return is_element(f) ? PNN_OK : (is_posit(f) || f == PNN_F64 ? PNN_EUNSUPPORTED : PNN_EINVAL); }
inline int kind_of(int f) { return f == PNN_F32 ? KIND_F32 : (f == PNN_BF16 ? KIND_BF16 : (elem_size(f) == 1 ? KIND_POSIT_U8 : KIND_POSIT_U16)); }
inline size_t element_bytes(int f) { return f == PNN_BF16 ? 2 : elem_size(f); }
inline ElemFmt elem_fmt(int f) {
    ElemFmt e = {16, 0};
    if (is_posit(f)) fmt_params(f, e.n, e.es);
    return e;
}

// Threads of a launch along x are counted in 32 bits: of more, some workgroups run and no error is reported.  Most workgroups of that many threads:
constexpr int64_t most_workgroups(int threads) { return 0xFFFFFFFFll / threads; }

PNN_HD float f32_of_bits(uint32_t b) { return __builtin_bit_cast(float, b); }
PNN_HD uint32_t bits_of_f32(float v) { return __builtin_bit_cast(uint32_t, v); }

// A posit's magnitude pattern and its value are tied by one integer:  T = k 2^(23+es) + (exponent and fraction, 23 + es bits)  is the
// binary32 word of the value less that of 1.  Two facts make both directions short:
//  - negating the n-1 bits of the pattern negates T (regime ones become zeros, what follows its complement), so only values
//    below 1 need to be handled: their regime is a run of zeros and its terminating one;
//  - that is how an integer looks to the conversion between integers and binary32: converting the pattern to binary32
//    counts the run and puts exponent and fraction at the top of the significand, adding 2^23 to a binary32 puts a significand behind
//    a run of zeros and rounds it, nearest with ties to even.

//
// The parts of both directions that leave zero and NaR (NaN) aside:

// Value; 0 and NaR give garbage and y == 0.  A negative pattern needs no negation: without its sign it is the negated magnitude, so T changes sign.
PNN_HD float posit_value_regular(uint32_t p, ElemFmt f, uint32_t& y) {
    const uint32_t u = p << (32 - f.n), x = u << 1;             // sign on top; regime on top; zeros below the pattern
    y = (uint32_t)((int32_t)x < 0 ? 0 - x : x);
    const uint32_t t = (bits_of_f32((float)y) << f.es) - (158u << (23 + f.es));
    const uint32_t s = (uint32_t)((int32_t)(x ^ u) >> 31);
    const uint32_t mag = (t ^ s) + ((127u << 23) - s);
    return f32_of_bits((mag & 0x7FFFFFFFu) | (u & 0x80000000u));
}

// Nearest pattern, in the low n bits, for a finite nonzero value; `value` receives what it stands for.
template <bool VALUE>
PNN_HD uint32_t posit_nearest_regular(float v, ElemFmt f, float& value) {
    const uint32_t bits = bits_of_f32(v), t = (bits & 0x7FFFFFFFu) - (127u << 23), st = (uint32_t)((int32_t)t >> 31);
    const int32_t range = (int32_t)((uint32_t)((f.n - 2) << f.es) << 23);
    int32_t below = (int32_t)t < 0 ? (int32_t)t : -(int32_t)t;
    below = below > -range ? below : -range;
    // es bits leave the significand; they stay as "not zero" in its last ones, far below any cut
    const uint32_t g = (uint32_t)(below >> f.es) | ((uint32_t)below & ((1u << f.es) - 1u));
    // the rounded integer negated for a value of 1 and above, and for a negative one: as two's complement below 1.5 2^23
    const uint32_t exponent = (uint32_t)(127 + f.n - 2) << 23;
    const float cut = f32_of_bits(((g + exponent) & 0x7FFFFFFFu) | ((bits ^ ~t) & 0x80000000u)) + 12582912.f;
    if (VALUE) {
        const uint32_t r = ((bits_of_f32(cut - 12582912.f) & 0x7FFFFFFFu) - exponent) << f.es;
        const uint32_t mag = (r ^ ~st) + ((127u << 23) - ~st);
        value = f32_of_bits((mag & 0x7FFFFFFFu) | (bits & 0x80000000u));
    }
    return bits_of_f32(cut) ^ (~st & (1u << (f.n - 1)));
}

// Value of a posit of at most 16 bits, exact (at most 13 significant bits, |scale| <= 40); NaR gives NaN.
PNN_HD float posit_value(uint32_t p, ElemFmt f) {
    uint32_t y;
    const float v = posit_value_regular(p, f, y);
    return y == 0u ? f32_of_bits((p >> (f.n - 1)) & 1u ? 0x7FC00000u : 0u) : v;
}

// Nearest posit of at most 16 bits, ties to the even pattern, never zero or NaR for a finite nonzero value; NaN and infinities
// give NaR.  `value` receives what the pattern stands for.
template <bool VALUE>
PNN_HD uint32_t posit_nearest(float v, ElemFmt f, float& value) {
    const uint32_t p = posit_nearest_regular<VALUE>(v, f, value) & ((1u << f.n) - 1u), ah = bits_of_f32(v) & 0x7FFFFFFFu;
    const bool zero = ah == 0u, nar = ah >= 0x7F800000u;
    if (VALUE) value = zero ? 0.f : (nar ? f32_of_bits(0x7FC00000u) : value);
    return zero ? 0u : (nar ? 1u << (f.n - 1) : p);
}
PNN_HD uint32_t posit_nearest(float v, ElemFmt f) {
    float none;
    return posit_nearest<false>(v, f, none);
}

// ---- in memory ----
template <int K> struct Raw;
template <> struct Raw<KIND_POSIT_U8> { typedef uint8_t T; };
template <> struct Raw<KIND_POSIT_U16> { typedef uint16_t T; };
template <> struct Raw<KIND_BF16> { typedef uint16_t T; };
template <> struct Raw<KIND_F32> { typedef uint32_t T; };

template <int K>
PNN_HD float value_of(uint32_t raw, ElemFmt f) {
    if (K == KIND_F32) return f32_of_bits(raw);
    if (K == KIND_BF16) return f32_of_bits(raw << 16);
    return posit_value(raw, f);
}

template <int K>
PNN_HD uint32_t raw_of(float v, ElemFmt f) {
    if (K == KIND_F32) return bits_of_f32(v);
    if (K == KIND_BF16) return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v);
    return posit_nearest(v, f);
}

// kind known at run time (uniform): for operands that are few
PNN_HD float load_value(const void* p, int64_t i, int kind, ElemFmt f) {
    switch (kind) {
        case KIND_POSIT_U8: return posit_value(((const uint8_t*)p)[i], f);
        case KIND_POSIT_U16: return posit_value(((const uint16_t*)p)[i], f);
        case KIND_BF16: return f32_of_bits((uint32_t)((const uint16_t*)p)[i] << 16);
        default: return ((const float*)p)[i];
    }
}
PNN_HD void store_value(void* p, int64_t i, int kind, ElemFmt f, float v) {
    switch (kind) {
        case KIND_POSIT_U8: ((uint8_t*)p)[i] = (uint8_t)posit_nearest(v, f); break;
        case KIND_POSIT_U16: ((uint16_t*)p)[i] = (uint16_t)posit_nearest(v, f); break;
        case KIND_BF16: ((uint16_t*)p)[i] = (uint16_t)raw_of<KIND_BF16>(v, f); break;
        default: ((float*)p)[i] = v;
    }
}

// CALL sees `K`, the kind as a constant
#define PNN_DISPATCH_KIND(kind, CALL)                               \
    switch (kind) {                                                  \
        case KIND_POSIT_U8: { constexpr int K = KIND_POSIT_U8; CALL; } break;   \
        case KIND_POSIT_U16: { constexpr int K = KIND_POSIT_U16; CALL; } break; \
        case KIND_BF16: { constexpr int K = KIND_BF16; CALL; } break;           \
        default: { constexpr int K = KIND_F32; CALL; } break;                   \
    }

// ---- eight elements in a row, of a kind known at run time (uniform: the branches are the wave's) ----
// As they lie in memory, in a vector rather than an array: an array whose elements are taken under several conditions ends up in scratch
// memory.  Alignment is the element type's (wide loads and stores take any address here).
typedef uint32_t words8 __attribute__((ext_vector_type(8)));
typedef uint32_t words2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t words4_any __attribute__((ext_vector_type(4), aligned(1)));
struct Raw8 {
    words8 w;
};

__device__ __forceinline__ void load8(Raw8& r, const void* p, int64_t i, int kind, int left) {
    if (left >= 8) {
        if (kind == KIND_POSIT_U8) {
            const words2_any v = *(const words2_any*)((const uint8_t*)p + i);
            r.w.lo.lo = v;
        } else if (kind == KIND_F32) {
            const words4_any *const q = (const words4_any*)((const uint8_t*)p + 4 * i), v0 = q[0], v1 = q[1];
            r.w.lo = v0;
            r.w.hi = v1;
        } else {
            const words4_any v = *(const words4_any*)((const uint8_t*)p + 2 * i);
            r.w.lo = v;
        }
        return;
    }
    r.w = (words8)(0u);
    if (left <= 0) return;
    // the end of a row: all eight loads at once, of the first element in place of those behind the end (one load after the other, each behind a
    // condition, made a row of 5119 wait for seven memory latencies)
    uint32_t v[8];
    if (kind == KIND_POSIT_U8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = ((const uint8_t*)p)[i + (e < left ? e : 0)];
    } else if (kind == KIND_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = ((const uint32_t*)p)[i + (e < left ? e : 0)];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = ((const uint16_t*)p)[i + (e < left ? e : 0)];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? v[e] : 0u;
    if (kind == KIND_POSIT_U8) {
#pragma unroll
        for (int e = 0; e < 2; ++e) r.w[e] = v[4 * e] | v[4 * e + 1] << 8 | v[4 * e + 2] << 16 | v[4 * e + 3] << 24;
    } else if (kind == KIND_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.w[e] = v[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) r.w[e] = v[2 * e] | v[2 * e + 1] << 16;
    }
}

__device__ __forceinline__ uint32_t pattern8(const Raw8& r, int e, int kind) {
    return kind == KIND_POSIT_U8 ? (r.w[e / 4] >> (8 * (e & 3))) & 0xFFu : (e & 1 ? r.w[e / 2] >> 16 : r.w[e / 2] & 0xFFFFu);
}

__device__ __forceinline__ void values8(float (&v)[8], const Raw8& r, int kind, ElemFmt f) {
    if (kind == KIND_POSIT_U8 || kind == KIND_POSIT_U16) {
        // zeros and NaR are looked for once for all eight
        uint32_t least = 0xFFFFFFFFu;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t y;
            v[e] = posit_value_regular(pattern8(r, e, kind), f, y);
            least = y < least ? y : least;
        }
        if (least == 0u) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t p = pattern8(r, e, kind);
                v[e] = p == 0u ? 0.f : (p == 1u << (f.n - 1) ? f32_of_bits(0x7FC00000u) : v[e]);
            }
        }
    } else if (kind == KIND_BF16) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = f32_of_bits(e & 1 ? r.w[e / 2] & 0xFFFF0000u : r.w[e / 2] << 16);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = f32_of_bits(r.w[e]);
    }
}

// Rounds in place where VALUE (v receives what is stored).
template <bool VALUE>
__device__ __forceinline__ void raw8(Raw8& r, float (&v)[8], int kind, ElemFmt f) {
    if (kind == KIND_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.w[e] = bits_of_f32(v[e]);
    } else if (kind == KIND_BF16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            r.w[e] = raw_of<KIND_BF16>(v[2 * e], f) | raw_of<KIND_BF16>(v[2 * e + 1], f) << 16;
            if (VALUE) {
                v[2 * e] = f32_of_bits(r.w[e] << 16);
                v[2 * e + 1] = f32_of_bits(r.w[e] & 0xFFFF0000u);
            }
        }
    } else {
        uint32_t q[8], worst = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t odd = (bits_of_f32(v[e]) & 0x7FFFFFFFu) - 1u;  // zero, infinities and NaN: 0x7F7FFFFF and above
            worst = odd > worst ? odd : worst;
        }
        if (worst < 0x7F7FFFFFu) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float back = 0.f;
                q[e] = posit_nearest_regular<VALUE>(v[e], f, back);
                if (VALUE) v[e] = back;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float back = 0.f;
                q[e] = posit_nearest<VALUE>(v[e], f, back);
                if (VALUE) v[e] = back;
            }
        }
        if (kind == KIND_POSIT_U8) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
                r.w[e] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[4 * e + 3], q[4 * e + 2], 0x0C0C0400u), __builtin_amdgcn_perm(q[4 * e + 1], q[4 * e], 0x0C0C0400u), 0x05040100u);
        } else {
            const uint32_t mask = ((1u << f.n) - 1u) * 0x10001u;
#pragma unroll
            for (int e = 0; e < 4; ++e) r.w[e] = __builtin_amdgcn_perm(q[2 * e + 1], q[2 * e], 0x05040100u) & mask;
        }
    }
}

__device__ __forceinline__ void store8(void* p, int64_t i, const Raw8& r, int kind, int left) {
    if (left >= 8) {
        if (kind == KIND_POSIT_U8) {
            *(words2_any*)((uint8_t*)p + i) = r.w.lo.lo;
        } else if (kind == KIND_F32) {
            words4_any* const q = (words4_any*)((uint8_t*)p + 4 * i);
            q[0] = r.w.lo;
            q[1] = r.w.hi;
        } else {
            *(words4_any*)((uint8_t*)p + 2 * i) = r.w.lo;
        }
        return;
    }
    if (kind == KIND_POSIT_U8) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) ((uint8_t*)p)[i + e] = (uint8_t)(r.w[e / 4] >> (8 * (e & 3)));
    } else if (kind == KIND_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) ((uint32_t*)p)[i + e] = r.w[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) ((uint16_t*)p)[i + e] = (uint16_t)(r.w[e / 2] >> (16 * (e & 1)));
    }
}

// ---- sums and maxima over a wave, in a fixed order, in every lane ----
// Through the vector unit's own lane shifts (a shuffle through LDS takes ten times as long); the total arrives in lane 63.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lane_shift(uint32_t v, uint32_t none) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ float wave_sum(float v) {
#define PNN_STEP(CTRL, ROWS) v += f32_of_bits(lane_shift<CTRL, ROWS>(bits_of_f32(v), 0u));
    PNN_STEP(0x111, 0xF) PNN_STEP(0x112, 0xF) PNN_STEP(0x114, 0xF) PNN_STEP(0x118, 0xF) PNN_STEP(0x142, 0xA) PNN_STEP(0x143, 0xC)
#undef PNN_STEP
    return f32_of_bits((uint32_t)__builtin_amdgcn_readlane((int)bits_of_f32(v), 63));
}
__device__ __forceinline__ float wave_max(float v) {
#define PNN_STEP(CTRL, ROWS) v = fmaxf(v, f32_of_bits(lane_shift<CTRL, ROWS>(bits_of_f32(v), 0xFF800000u)));
    PNN_STEP(0x111, 0xF) PNN_STEP(0x112, 0xF) PNN_STEP(0x114, 0xF) PNN_STEP(0x118, 0xF) PNN_STEP(0x142, 0xA) PNN_STEP(0x143, 0xC)
#undef PNN_STEP
    return f32_of_bits((uint32_t)__builtin_amdgcn_readlane((int)bits_of_f32(v), 63));
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#define PNN_STEP(CTRL, ROWS) { const uint32_t o = lane_shift<CTRL, ROWS>(v, 0u); v = v > o ? v : o; }
    PNN_STEP(0x111, 0xF) PNN_STEP(0x112, 0xF) PNN_STEP(0x114, 0xF) PNN_STEP(0x118, 0xF) PNN_STEP(0x142, 0xA) PNN_STEP(0x143, 0xC)
#undef PNN_STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

}  // namespace pnn
