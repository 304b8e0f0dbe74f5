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
//    them up (AttnMarks) in what the packing kernel notes of the blocks that hold any.
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
typedef float at_v4f __attribute__((ext_vector_type(4)));
__device__ __forceinline__ at_v4f at_mfma16(at_v8b a, at_v8b b, at_v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
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
__device__ __forceinline__ bool at_sees(const AttnShape& s, int p, int low, int key) { return (key <= p) & ((key > low) | (key < s.sinks)); }

// Order of n tiles whose work falls with their number, for nbh heads each: back and forth over as many tiles as fill the chip's 256 compute
// units once, so that the workgroups that share a unit have about the same work together.
__device__ __forceinline__ int at_snake(int i, int n, int nbh) {
    const int lap = nbh < 256 ? 256 / nbh : 1, turn = i / lap, first = turn * lap, size = n - first < lap ? n - first : lap;
    return (turn & 1) ? first + size - 1 - (i - first) : i;
}

// What a block of 32 rows holds that is not finite: for each row, and last for all of them together, one bit an element of a head in three
// masks of 128 (+infinity, -infinity, NaN).
constexpr int AT_MARKS = 33 * 3;

// Of few queries: workgroups that a row block's keys are split over, what the kernel that joins them holds weights of.
constexpr int AT_MOST_PARTS = 256;

struct AttnPackItem {
    const void* src;
    int64_t sb, sl, sh;   // strides: batch, position, head
    int rows, blocks;
    uint4 *row_frags, *t_frags;  // either may be null
    int G, kind;
    ElemFmt f;
    int32_t* flags;       // one per block, may be null: whether it holds anything that is not finite
    uint4* marks;         // AT_MARKS per block, written where it does
};

struct AttnPack {
    AttnPackItem item[4];
    int B, HKV, D;
};

// 8 elements as bfloat16, exact for the formats accepted; zeros in place of those beyond `left`
__device__ __forceinline__ uint4 at_load8(const void* p, int64_t at, int left, int kind, ElemFmt f) {
    Raw8 r;
    load8(r, p, at, kind, left);
    if (kind == KIND_BF16) return make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
    float v[8];
    values8(v, r, kind, f);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(bits_of_f32(v[2 * i + 1]), bits_of_f32(v[2 * i]), 0x07060302u);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// whether either half of a word is an infinity or a NaN
__device__ __forceinline__ bool at_odd(uint32_t w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; }

// One block of 32 rows of one operand to a workgroup, through LDS.  Keys and values of 2 x 4001 x 4 heads of 128 in 8-bit posits: 13 us; of 4 x 2048, 16 heads on 4
// of 64, the seven operands of the backward pass 28.
template <int DB>
__global__ __launch_bounds__(256) void attn_pack_kernel(AttnPack a) {
    constexpr int DP = 32 * DB, KS = 2 * DB;
    __shared__ uint16_t tile[32][DP + 2];
    uint32_t* const words = (uint32_t*)&tile[0][0];
    const int n = blockIdx.z / a.B, b = blockIdx.z - n * a.B, hk = blockIdx.y, t = threadIdx.x;
    const AttnPackItem& p = a.item[n];
    const int blk = blockIdx.x;
    if (blk >= p.blocks) return;
    bool odd = false;
    for (int c = t; c < 32 * DP / 8; c += 256) {
        const int r = c / (DP / 8), d = (c - r * (DP / 8)) * 8;
        const int row = blk * 32 + r;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < p.rows && d < a.D) {
            const int i = row / p.G, g = row - i * p.G;
            v = at_load8(p.src, b * p.sb + i * p.sl + (int64_t)(hk * p.G + g) * p.sh + d, a.D - d, p.kind, p.f);
        }
        uint32_t* const to = words + r * (DP / 2 + 1) + d / 2;
        to[0] = v.x;
        to[1] = v.y;
        to[2] = v.z;
        to[3] = v.w;
        odd |= at_odd(v.x) || at_odd(v.y) || at_odd(v.z) || at_odd(v.w);
    }
    const bool any = __syncthreads_or(odd);
    const int64_t bh = (int64_t)b * a.HKV + hk;
    if (p.flags && t == 0) p.flags[bh * p.blocks + blk] = any;
    if (p.flags && any) {
        // a row to a thread and word of 32 elements, then the columns' together
        uint32_t* const m = (uint32_t*)(p.marks + (bh * p.blocks + blk) * AT_MARKS);
        for (int c = t; c < 32 * 4; c += 256) {
            const int r = c >> 2, d = c & 3;
            uint32_t pos = 0, neg = 0, nan = 0;
            for (int e = 0; d < DB && e < 32; ++e) {
                const uint32_t x = tile[r][d * 32 + e], bit = (x & 0x7F80u) == 0x7F80u ? 1u << e : 0u;
                nan |= x & 0x7Fu ? bit : 0u;
                neg |= (x & 0x807Fu) == 0x8000u ? bit : 0u;
                pos |= (x & 0x807Fu) == 0u ? bit : 0u;
            }
            m[r * 12 + d] = pos;
            m[r * 12 + 4 + d] = neg;
            m[r * 12 + 8 + d] = nan;
        }
        __syncthreads();
        if (t < 12) {
            uint32_t w = 0;
            for (int r = 0; r < 32; ++r) w |= m[r * 12 + t];
            m[32 * 12 + t] = w;
        }
    }
    if (p.row_frags)
        for (int c = t; c < KS * 64; c += 256) {
            const int l = c & 63, r = l & 31, d = (c >> 6) * 16 + 8 * (l >> 5);
            const uint32_t* const w = words + r * (DP / 2 + 1) + d / 2;
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
    const at_v4u w = __builtin_bit_cast(at_v4u, hi);
    at_v8b o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o[2 * i] = (__bf16)(v[from + 2 * i] - f32_of_bits(w[i] << 16));
        o[2 * i + 1] = (__bf16)(v[from + 2 * i + 1] - f32_of_bits(w[i] & 0xFFFF0000u));
    }
    return o;
}

// v.x of lanes 32 .. 63 and v.y of lanes 0 .. 31 change places
__device__ __forceinline__ void at_swap_halves(float& x, float& y) {
    typedef uint32_t v2 __attribute__((ext_vector_type(2)));
    const v2 r = __builtin_amdgcn_permlane32_swap(bits_of_f32(x), bits_of_f32(y), false, false);
    x = f32_of_bits(r.x);
    y = f32_of_bits(r.y);
}
// the larger of a lane's value and that of the lane 32 away
__device__ __forceinline__ float at_max_halves(float v) {
    float w = v;
    at_swap_halves(v, w);
    return fmaxf(v, w);
}
// A block's 32 elements of the lane's row, 8 in a row at a time: f(first of them, values).  The halves of a wave hold the same rows; each takes
// every other eight.
template <class F>
__device__ __forceinline__ void at_eights(const at_v16f& v, int half, F f) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = v[8 * q + i];
            x[4 + i] = v[8 * q + 4 + i];
            at_swap_halves(x[i], x[4 + i]);
        }
        f(8 * (2 * q + half), x);
    }
}
__device__ __forceinline__ void at_store8(void* p, int64_t at, int left, int kind, ElemFmt f, const float (&v)[8]) {
    if (left <= 0) return;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = v[i];
    Raw8 r;
    raw8<false>(r, w, kind, f);
    store8(p, at, r, kind, left);
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

// What infinities and NaN that a result's row (its key, in the backward pass) sees make of it; the packed operand held zeros in their place.
template <int DB>
struct AttnMarks {
    uint32_t pos[DB], neg[DB], nan[DB];  // one bit an element of a head
    __device__ __forceinline__ void add(const uint32_t (&p)[4], const uint32_t (&n)[4], const uint32_t (&q)[4], bool see) {
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            pos[d] |= see ? p[d] : 0u;
            neg[d] |= see ? n[d] : 0u;
            nan[d] |= see ? q[d] : 0u;
        }
    }
    // the three masks of a block's row, as the packing kernel left them
    __device__ __forceinline__ void add(const uint4* m, bool see) {
        uint32_t w[3][4];
        __builtin_memcpy(w, m, sizeof w);
        add(w[0], w[1], w[2], see);
    }
    // the marks of all lanes together, in every lane; `see`: whether the lane's row has them
    __device__ __forceinline__ void add_all_lanes(const AttnMarks& o, bool see) {
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            uint32_t w[3] = {o.pos[d], o.neg[d], o.nan[d]};
#pragma unroll
            for (int x = 0; x < 3; ++x) {
                for (int m = 32; m >= 1; m >>= 1) w[x] |= (uint32_t)__shfl_xor((int)w[x], m, 64);
                w[x] = see ? w[x] : 0u;
            }
            pos[d] |= w[0];
            neg[d] |= w[1];
            nan[d] |= w[2];
        }
    }
};
// v, given the three masks' words that its bit is in
__device__ __forceinline__ float at_marked(float v, uint32_t pos, uint32_t neg, uint32_t nan, int bit) {
    const bool p = (pos >> bit) & 1u, n = (neg >> bit) & 1u;
    if (((nan >> bit) & 1u) || (p && n) || v != v) return f32_of_bits(0x7FC00000u);
    return p ? f32_of_bits(0x7F800000u) : (n ? f32_of_bits(0xFF800000u) : v);
}

// How the 32 rows of a wave see a block of 32 of the other side: not at all, all of them all of it, only where `sink` says so, or each pair for itself.
enum AttnSight { AT_NONE, AT_ALL, AT_SINKS, AT_EDGE };

// Marks of `count` blocks for a wave's rows; all its lanes call.  Blocks seen alike are taken one to a lane, those at the mask's edges row by row: as
// many as the mask has edges, whatever the length.
template <int DB, class Block, class Sight, class Sees>
__device__ __forceinline__ AttnMarks<DB> at_marks(const int32_t* flags, const uint4* marks, int count, bool sink, Block block, Sight sight, Sees sees) {
    AttnMarks<DB> own = {}, all = {}, sinks = {};
    const int lane = threadIdx.x & 63;
    for (int n0 = 0; n0 < count; n0 += 64) {
        const bool in = n0 + lane < count;
        const int blk = in ? block(n0 + lane) : 0, how = in && flags[blk] ? sight(blk) : AT_NONE;
        if (how == AT_ALL) all.add(marks + (int64_t)blk * AT_MARKS + 96, true);
        if (how == AT_SINKS) sinks.add(marks + (int64_t)blk * AT_MARKS + 96, true);
        for (uint64_t edge = __ballot(how == AT_EDGE); edge; edge &= edge - 1) {
            const int at = block(n0 + __builtin_ctzll(edge));
#pragma unroll 4
            for (int r = 0; r < 32; ++r) own.add(marks + (int64_t)at * AT_MARKS + 3 * r, sees(at * 32 + r));
        }
    }
    own.add_all_lanes(all, true);
    own.add_all_lanes(sinks, sink);
    return own;
}

}  // namespace pnn
