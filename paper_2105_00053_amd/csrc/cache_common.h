// A cache of keys and values in pages: where its elements lie, and its format of 4 bits.
//
// A page of one head is one run of memory, keys as [token][D] and values as [token / 4][D / 8][token % 4][8]: the lanes of attention read whole runs of both, of
// values four tokens' eight elements at once, which they need side by side.  4-bit floats are two to a byte, with the blocks' powers in the same order behind them.
#pragma once

#include "heads_common.h"

namespace pnn {

enum CacheKind { CACHE_U8 = 0, CACHE_BF16 = 1, CACHE_F4 = 2 };

struct CacheShape {
    int B, HKV, D, blocks;  // blocks of 32 elements in a head
    int page, shift, pages, columns;
    int64_t pitch, bytes;   // of a page of one head
    const int32_t *starts, *lens, *table;
    int T;
};

inline bool is_cache_format(int f) { return f == PNN_F4 || f == PNN_BF16 || (is_posit(f) && elem_size(f) == 1); }
inline int cache_format_status(int f) { return is_cache_format(f) ? PNN_OK : (is_posit(f) || is_float(f) ? PNN_EUNSUPPORTED : PNN_EINVAL); }
inline int cache_kind(int f) { return f == PNN_F4 ? CACHE_F4 : (f == PNN_BF16 ? CACHE_BF16 : CACHE_U8); }

// What append, read and attention ask of a description alike
inline int paged_status(const pnn_paged_desc* d) {
    if (!d || d->T < 0 || d->B < 0 || d->HQ < 0 || d->HKV < 0 || d->D < 0 || d->page <= 0 || d->pages < 0 || d->columns < 0 || d->pitch < d->columns) return PNN_EINVAL;
    if ((d->page & (d->page - 1)) != 0 || d->page < 16 || d->page > 4096 || d->D % 8 != 0 || d->D > 128) return PNN_EUNSUPPORTED;
    const int64_t most = (int64_t)1 << 31;
    if (d->T >= most || d->B >= 65536 || d->HQ >= 65536 || d->HKV >= 65536 || d->pages >= most || d->columns * d->page >= most - 128) return PNN_EUNSUPPORTED;
    return PNN_OK;
}

inline CacheShape cache_shape(const pnn_paged_desc& d, int fcache, const int32_t* starts, const int32_t* lens, const int32_t* table) {
    CacheShape s;
    s.B = (int)d.B; s.HKV = (int)d.HKV; s.D = (int)d.D; s.blocks = (int)((d.D + 31) / 32);
    s.page = (int)d.page; s.shift = __builtin_ctzll((unsigned long long)d.page); s.pages = (int)d.pages; s.columns = (int)d.columns;
    s.pitch = d.pitch;
    s.bytes = fcache == PNN_F4 ? d.page * (d.D / 2 + s.blocks) : d.page * d.D * (int64_t)element_bytes(fcache);
    s.starts = starts; s.lens = lens; s.table = table;
    s.T = (int)d.T;
    return s;
}

// First of a sequence's rows and the row behind its last, within 0 .. T
__device__ __forceinline__ int cache_first(const CacheShape& s, int b) {
    const int v = s.starts ? s.starts[b] : b;
    return v < 0 ? 0 : (v > s.T ? s.T : v);
}
// A page of a head: its first byte, null where `column` is none of the sequence's or its entry no page
__device__ __forceinline__ int64_t cache_page(const CacheShape& s, int b, int column, int h) {
    if (column < 0 || column >= s.columns) return -1;
    const int p = s.table[b * s.pitch + column];
    return p < 0 || p >= s.pages ? -1 : ((int64_t)p * s.HKV + h) * s.bytes;
}
// Element, from a page's first, of eight elements `unit` of the token at `at`
__device__ __forceinline__ int cache_unit(const CacheShape& s, bool values, int at, int unit) {
    return values ? (((at >> 2) * (s.D >> 3) + unit) * 4 + (at & 3)) * 8 : at * s.D + unit * 8;
}
// Of a value, the unit that a lane of 16 takes in attention, where a head is DB blocks of 32 (`full`: whole ones): the lanes share out 64 elements, or 128, and those behind the head's
// end, which 32 and 96 elements leave too, take its first unit
__host__ __device__ constexpr int cache_lane_unit(int DB, bool full, int col, int D) {
    const int unit = (DB <= 2 ? 4 : 8) * col / 8;
    return (full && (DB == 2 || DB == 4)) || unit < D / 8 ? unit : 0;
}
// Byte, from a page's first, of a block's power
__device__ __forceinline__ int cache_power(const CacheShape& s, bool values, int at, int block) {
    return s.page * s.D / 2 + (values ? ((at >> 2) * s.blocks + block) * 4 + (at & 3) : at * s.blocks + block);
}

// A block's power, as its byte, from its largest magnitude's binary32 word: the smallest that leaves that at 7 or below
__device__ __forceinline__ uint32_t f4_power(uint32_t most) {
    int e = (int)(most >> 23) - 2 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    e = e < 3 ? 3 : (e > 252 ? 252 : e);
    return most >= 0x7F800000u ? 255u : (uint32_t)e;
}
__device__ __forceinline__ float f4_scale(uint32_t power) { return f32_of_bits(power << 23); }
// Eight elements' codes: over the block's power, to nearest, ties to the even code, 6 for what is above it
__device__ __forceinline__ uint32_t f4_codes(const float (&v)[8], uint32_t power) {
    const float s = f4_scale(power);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
}
// Eight elements of 4 bits
__device__ __forceinline__ void f4_values(float (&v)[8], uint32_t w, uint32_t power) {
    typedef float v2 __attribute__((ext_vector_type(2)));
    const float s = f4_scale(power);
    const v2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
    const v2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
    v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
    if (power == 255u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = f32_of_bits(0x7FC00000u);
    }
}

}  // namespace pnn
