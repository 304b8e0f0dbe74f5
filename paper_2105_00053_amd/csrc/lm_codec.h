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

PNN_HD float f32_of_bits(uint32_t b) { return __builtin_bit_cast(float, b); }
PNN_HD uint32_t bits_of_f32(float v) { return __builtin_bit_cast(uint32_t, v); }

// Value of a posit of at most 16 bits (exact: at most 13 significant bits, |scale| <= 40).  Regime, exponent and fraction are one
// string; with the regime's k taken off, what is left is exponent and fraction as binary32 has them, shifted.
PNN_HD float posit_value(uint32_t p, ElemFmt f) {
    const int32_t u = (int32_t)(p << (32 - f.n));               // sign on top; zeros below the pattern
    const uint32_t a = (uint32_t)(u < 0 ? 0 - (uint32_t)u : (uint32_t)u);
    const uint32_t x = a << 1;                                   // regime on top
    const uint32_t ones = (uint32_t)((int32_t)x >> 31);
    const uint32_t run = (uint32_t)clz32(x ^ ones);              // run length (the bit behind the pattern ends it at the latest)
    const uint32_t k = (run ^ ~ones) + 1u + 2u * ones;           // run - 1 or -run
    const uint32_t rest = (x << (run & 31u)) << 1;               // exponent, then fraction
    const uint32_t mag = ((127u + (k << f.es)) << 23) + (rest >> (9 - f.es));
    const uint32_t v = mag | ((uint32_t)u & 0x80000000u);
    return f32_of_bits((uint32_t)u == 0x80000000u ? 0x7FC00000u : (u == 0 ? 0u : v));
}

// Nearest posit of at most 16 bits, ties to the even pattern, never zero or NaR for a finite nonzero value; NaN and infinities
// give NaR.  The string regime | exponent | fraction comes from an arithmetic right shift of "10" in front of exponent and fraction (for
// a negative k everything complemented); fraction bits that the cut cannot reach are folded into one that no shift pushes out.
PNN_HD uint32_t posit_nearest(float v, ElemFmt f) {
    const uint32_t bits = bits_of_f32(v);
    const uint32_t ah0 = bits & 0x7FFFFFFFu;
    const uint32_t range = (uint32_t)((f.n - 2) << f.es) << 23, one = 127u << 23;
    const uint32_t low = ah0 < one - range ? one - range : ah0;
    const uint32_t h = (low > one + range ? one + range : low) - one;
    const int k = (int32_t)h >> (23 + f.es);
    const uint32_t sg = (uint32_t)(k >> 31);
    const uint32_t kk = (uint32_t)k ^ sg;
    uint32_t tail = h << (9 - f.es);
    const uint32_t reach = 1u << f.n;                            // bits of the tail below this one lie behind every cut
    tail |= (tail & (reach - 1u)) ? reach : 0u;
    const uint32_t w = 0x80000000u | ((tail ^ sg) >> 2);
    const uint32_t x = (uint32_t)((int32_t)w >> kk) ^ sg;
    const int cut = 33 - f.n;
    const uint32_t lsb = (x >> cut) & 1u;
    const uint32_t body = (x + ((1u << (cut - 1)) - 1u) + lsb) >> cut;
    const uint32_t sm = (uint32_t)((int32_t)bits >> 31);
    const uint32_t mask = (1u << f.n) - 1u;
    const uint32_t p = ((body ^ sm) - sm) & mask;
    return ah0 == 0u ? 0u : (ah0 >= 0x7F800000u ? 1u << (f.n - 1) : p);
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

// ---- sums over a workgroup, in a fixed order ----
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor(v, m, 64));
    return v;
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)v, m, 64);
        v = v > o ? v : o;
    }
    return v;
}

}  // namespace pnn
