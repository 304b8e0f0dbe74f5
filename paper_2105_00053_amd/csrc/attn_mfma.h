// What the attention kernels share: bfloat16 matrix instructions, operands rewritten once in their lane order, and the packing kernel.
//
// v_mfma_f32_32x32x16_bf16: lane l holds, for A, row l % 32 and the 8 reduction indices from 8 (l / 32); for B, column l % 32 and the same
// indices; result register r is row (r % 4) + 8 (r / 4) + 4 (l / 32), column l % 32.  The order of the reduction indices is free as long
// as both operands use the same one, which two things here rest on:
//  - "row fragments" hold 32 rows x 16 of a head's elements: the operands of the products that reduce over a head's elements;
//  - "transposed fragments" hold 32 of a head's elements x 16 rows, the rows in the order (l / 32, i) -> 4 (l / 32) + i for i < 4, else
//    8 + 4 (l / 32) + i - 4: the order in which a lane's result registers hold them.  So the probabilities of one product are operands
//    of the next as they come out of it, rounded in place, without any exchange between lanes.  They hold zeros in place of infinities and
//    NaN: a probability of zero times one of those would reach rows that do not see it.  Where they matter the kernels look
//    them up (AttnMarks) in blocks that the packing kernel flagged.
// Formats that bfloat16 holds exactly make every product exact; decoding in the kernels themselves would cost 14 vector operations an element
// and tile, four times what the matrix instructions of a tile of 128 x 64 take, so each operand is decoded once.
// The query heads that share a key head are one operand: row r = position * G + head within the group.
#pragma once

#include "lm_codec.h"

namespace pnn {

typedef float at_v16f __attribute__((ext_vector_type(16)));
typedef __bf16 at_v8b __attribute__((ext_vector_type(8)));
typedef uint32_t at_v4u __attribute__((ext_vector_type(4)));

__device__ __forceinline__ at_v16f at_mfma(at_v8b a, at_v8b b, at_v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ at_v8b at_frag(const uint4& v) { return __builtin_bit_cast(at_v8b, v); }
__device__ __forceinline__ at_v16f at_zero() {
    at_v16f z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    return z;
}
// row of result register r for the lane's half
__device__ __forceinline__ int at_row(int r, int half) { return (r & 3) + 8 * (r >> 2) + 4 * half; }

// A wave's 1 KB run from memory straight into LDS, 16 bytes a lane.
__device__ __forceinline__ void at_copy(const uint4* src, uint4* dst, int lane) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + lane), (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}
// This wave's copies have landed; behind the barrier everyone's have, and everyone's reads of the other buffer are done.
__device__ __forceinline__ void at_landed() {
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    __syncthreads();
}

// Positions, rows and blocks of one sequence fit 32 bits; offsets into tensors do not.
struct AttnShape {
    int LQ, LK;
    int window, sinks;      // window 0: none, which any of LK keys or more is; sinks at most LK
    int rows;               // LQ * G
    int qblocks, kblocks;   // blocks of 32 rows / keys in the packed operands, multiples of 4
    const int32_t* lens;
    int HKV, G, D;
    float scale;
};

__device__ __forceinline__ int at_keys(const AttnShape& s, int64_t b) {
    const int n = s.lens ? s.lens[b] : s.LK;
    return n < 0 ? 0 : (n > s.LK ? s.LK : n);
}
// whether a query at position p sees a key; low = the last position in front of its window
__device__ __forceinline__ bool at_sees(const AttnShape& s, int p, int low, int key) { return key <= p && (key > low || key < s.sinks); }

struct AttnPackItem {
    const void* src;
    int64_t sb, sl, sh;   // strides: batch, position, head
    int rows, blocks;
    uint4 *row_frags, *t_frags;  // either may be null
    int G, kind;
    ElemFmt f;
    int32_t* flags;       // one per block, may be null: whether it holds anything that is not finite
};

struct AttnPack {
    AttnPackItem item[4];
    int B, HKV, D;
};

// 8 elements as bfloat16, exact for the formats accepted
template <int K>
__device__ __forceinline__ void at_load8(const void* p, int64_t at, int left, ElemFmt f, uint16_t (&o)[8]) {
    typedef typename Raw<K>::T T;
    const T* s = (const T*)p + at;
    T raw[8];
    if (left >= 8) {
        __builtin_memcpy(raw, s, 8 * sizeof(T));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[i] = i < left ? s[i] : (T)0;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (uint16_t)(bits_of_f32(value_of<K>(raw[i], f)) >> 16);
}

// One block of 32 rows of one operand to a workgroup, through LDS.
template <int DB>
__global__ __launch_bounds__(256) void attn_pack_kernel(AttnPack a) {
    constexpr int DP = 32 * DB, KS = 2 * DB;
    __shared__ uint16_t tile[32][DP + 2];
    const int n = blockIdx.z / a.B, b = blockIdx.z - n * a.B, hk = blockIdx.y, t = threadIdx.x;
    const AttnPackItem& p = a.item[n];
    const int blk = blockIdx.x;
    if (blk >= p.blocks) return;
    bool odd = false;
    for (int c = t; c < 32 * DP / 8; c += 256) {
        const int r = c / (DP / 8), d = (c - r * (DP / 8)) * 8;
        const int row = blk * 32 + r;
        uint16_t v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (row < p.rows && d < a.D) {
            const int i = row / p.G, g = row - i * p.G;
            const int64_t at = b * p.sb + i * p.sl + (int64_t)(hk * p.G + g) * p.sh + d;
            if (p.kind == KIND_POSIT_U8) at_load8<KIND_POSIT_U8>(p.src, at, a.D - d, p.f, v);
            else if (p.kind == KIND_POSIT_U16) at_load8<KIND_POSIT_U16>(p.src, at, a.D - d, p.f, v);
            else at_load8<KIND_BF16>(p.src, at, a.D - d, p.f, v);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            tile[r][d + i] = v[i];
            odd |= (v[i] & 0x7F80u) == 0x7F80u;
        }
    }
    const bool any = __syncthreads_or(odd);
    const int64_t bh = (int64_t)b * a.HKV + hk;
    if (p.flags && t == 0) p.flags[bh * p.blocks + blk] = any;
    if (p.row_frags)
        for (int c = t; c < KS * 64; c += 256) {
            const int l = c & 63, r = l & 31, d = (c >> 6) * 16 + 8 * (l >> 5);
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (uint32_t)tile[r][d + 2 * i] | ((uint32_t)tile[r][d + 2 * i + 1] << 16);
            p.row_frags[(bh * p.blocks + blk) * KS * 64 + c] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    if (p.t_frags)
        for (int c = t; c < 2 * DB * 64; c += 256) {
            const int l = c & 63, q = c >> 6, k0 = (q / DB) * 16 + 4 * (l >> 5), d = (q % DB) * 32 + (l & 31);
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t x[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int e = 2 * i + j;
                    x[j] = tile[k0 + (e < 4 ? e : e + 4)][d];
                    if ((x[j] & 0x7F80u) == 0x7F80u) x[j] = 0;
                }
                w[i] = x[0] | (x[1] << 16);
            }
            p.t_frags[(bh * p.blocks + blk) * 2 * DB * 64 + c] = make_uint4(w[0], w[1], w[2], w[3]);
        }
}

// eight result registers as an operand, rounded to bfloat16
__device__ __forceinline__ at_v8b at_round(const at_v16f& v, int from) {
    at_v8b o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)v[from + i];
    return o;
}
// what that rounding left, rounded in turn: together 16 bits
__device__ __forceinline__ at_v8b at_rest(const at_v16f& v, int from, const at_v8b& hi) {
    at_v8b o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)(v[from + i] - (float)hi[i]);
    return o;
}

// The scale of the scores, as what exp2 takes: kept positive, so that the largest score has the largest exponent; its sign goes into q, and where it
// is zero q does (a NaN in it stays one).
__device__ __forceinline__ float at_scale(float c) { return c < 0.f ? -c : (c == 0.f ? 1.f : c); }
__device__ __forceinline__ at_v8b at_scaled(uint4 v, float c) {
    if (c < 0.f) v = make_uint4(v.x ^ 0x80008000u, v.y ^ 0x80008000u, v.z ^ 0x80008000u, v.w ^ 0x80008000u);
    at_v8b q = at_frag(v);
    if (c == 0.f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = (__bf16)((float)q[e] * 0.f);
    }
    return q;
}

// What infinities and NaN that a result's row sees make of it; the packed operand held zeros in their place.
struct AttnMarks {
    uint32_t pos[2], neg[2], nan[2];  // one bit a result register
    __device__ __forceinline__ void add(int bit, float v) {
        const uint32_t m = 1u << (bit & 31);
        const bool hi = bit >= 32, inf = v - v != 0.f && v == v;
        const uint32_t p = inf && v > 0.f ? m : 0u, n = inf && v < 0.f ? m : 0u, x = v != v ? m : 0u;
        if (hi) { pos[1] |= p; neg[1] |= n; nan[1] |= x; }
        else { pos[0] |= p; neg[0] |= n; nan[0] |= x; }
    }
    __device__ __forceinline__ float apply(int bit, float v) const {
        const int k = bit >> 5, sh = bit & 31;
        const bool p = (pos[k] >> sh) & 1u, n = (neg[k] >> sh) & 1u;
        if (((nan[k] >> sh) & 1u) || (p && n) || v != v) return f32_of_bits(0x7FC00000u);
        return p ? f32_of_bits(0x7F800000u) : (n ? f32_of_bits(0xFF800000u) : v);
    }
};

}  // namespace pnn
