// Attention of a few new tokens on a cache in pages.
//
// A workgroup takes 16 rows (positions and heads of a group) of a sequence and a part of the keys that they see; its four waves take tiles of 32 keys in turn, as the kernel of
// attn_token.h does, whose matrix instructions and orders these are: S^T = K Q^T, then O^T += V^T P^T with the probabilities as they come out of the first product.
// What differs is where elements come from.  The order of a head's elements in the first product is free, so a lane takes a run of a key's elements (8 for each block of 32), and a
// page holds four tokens' values side by side, so that a lane's eight values of a block of elements are two runs.  Page numbers are looked up one tile ahead of the loads that need them.
// 4-bit floats become bfloat16 two at a time with their block's power, in one instruction; 8-bit posits through a table in LDS that every bank has a copy of.
#pragma once

#include "attn_prompt.h"
#include "cache_common.h"

namespace pnn {

struct AttnPaged {
    CacheShape s;
    AttnShape n;          // window, sinks, G, D, scale, LK: the longest
    const void* q;
    const char *k, *v;
    int64_t ql, qh;
    int kq, most;
    ElemFmt fq, fc;
    void* o;
    float* lse;
    int ko;
    ElemFmt fo;
    int rows, blocks;     // of a row block; row blocks
    int tiles, parts;     // of a part; workgroups that a row block's keys are split over
    float* part;          // [row block][part][m: rows][l: rows][rows][D]
};

// A sequence's rows and keys
struct PagedRows {
    int first, count, rows, keys, base;  // rows: those of the heads of a group; base: the first one's position
    __device__ __forceinline__ PagedRows(const AttnPaged& a, int b) {
        first = cache_first(a.s, b);
        const int end = a.s.starts ? cache_first(a.s, b + 1) : b + 1;
        count = end > first ? end - first : 0;
        const int n = a.s.lens[b];
        keys = n < 0 ? 0 : (n > a.n.LK ? a.n.LK : n);
        base = keys - count;
        rows = (count < a.most ? count : a.most) * a.n.G;
    }
};

// A tile's keys and values as they lie in memory
template <int KC, int KS>
struct PagedRaw {
    static constexpr int KW = KC == CACHE_F4 ? 1 : (KC == CACHE_U8 ? 2 : 4);  // words of eight elements
    uint32_t k[2][KS * KW], v[2][4 * KW];
    uint32_t kp[2][KC == CACHE_F4 ? KS : 1], vp[KC == CACHE_F4 ? 2 : 1];  // powers
    bool bad[2];  // the halves' pages are none
};

// Of a value that stands in the lanes N further up in the row of 16, or down (zero where there is none)
template <int N>
__device__ __forceinline__ uint32_t from_above(uint32_t v) { return lane_shift<0x100 + N, 0xF>(v, 0u); }
// v of the lane's row N further down in the banks (of four lanes) of BANKS, `own` elsewhere
template <int N, int BANKS>
__device__ __forceinline__ float spread(float own, float v) {
    return f32_of_bits((uint32_t)__builtin_amdgcn_update_dpp((int)bits_of_f32(own), (int)bits_of_f32(v), 0x110 + N, 0xF, BANKS, false));
}
template <int N>
__device__ __forceinline__ float turned(float v) { return f32_of_bits(lane_shift<0x120 + N, 0xF>(bits_of_f32(v), 0u)); }
// the larger of a lane's value and that of the lane 16 away
__device__ __forceinline__ float max_rows(float v) {
    typedef uint32_t v2 __attribute__((ext_vector_type(2)));
    const v2 r = __builtin_amdgcn_permlane16_swap(bits_of_f32(v), bits_of_f32(v), false, false);
    return fmaxf(f32_of_bits(r.x), f32_of_bits(r.y));
}

// Bound by memory where lengths are alike (64 x 8192, 32 heads on 8 of 128, 4 bits: 571 MB in 126 us, 4.5 TB/s), by the longest's end where not (the same up to 8192: 83 us with its join), by the chain of table, loads,
// products and joins where keys are few (3 x 300: 8.8 us).  Of 4 rows to a group the shared scores made 94 us of 155.
// ROWS: of a block (4, 8 or 16).  The first product has 16 columns, one to a lane of 16, and four lanes have a column; of fewer rows the scores go to the lanes whose columns
// are none, so that each works on 8 ROWS / 16 of them.  FULL: heads of 32 DB elements.
template <int KC, int DB, int ROWS, bool FULL>
__global__ __launch_bounds__(256, KC == CACHE_BF16 ? 2 : 3) void attn_paged_kernel(AttnPaged a) {
    constexpr int KS = DB, NV = DB <= 2 ? 4 : 8, SC = ROWS / 2;
    typedef PagedRaw<KC, KS> R;
    __shared__ uint32_t smem[8192];  // the table, then what the waves join through
    __shared__ float wm[4][16], wl[4][16];
    const CacheShape& s = a.s;
    const AttnShape& n = a.n;
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), quarter = lane >> 4, col = lane & 15;
    // Heads fastest, then sequences, row blocks, parts: the later parts, which the longer sequences alone have, spread over the chip's eight dies as all others do (with parts fastest, four
    // of them left two dies without work: 64 sequences of up to 8192 took 104 us where three took 85), and short ones come last.
    const unsigned heads = (unsigned)s.HKV, groups = heads * s.B;
    const int part = blockIdx.x / (groups * a.blocks), rb = blockIdx.x / groups % a.blocks, b = blockIdx.x % groups / heads, hk = blockIdx.x % heads;
    const PagedRows x(a, b);
    if (rb * ROWS >= x.rows) return;
    const int row = rb * ROWS + col % ROWS, last = rb * ROWS + ROWS - 1 < x.rows ? rb * ROWS + ROWS - 1 : x.rows - 1;
    const int i = row / n.G, h = hk * n.G + (row - i * n.G);
    const bool live = row < x.rows;
    const int p = live ? x.base + i : -1, low = n.window ? p - n.window : -1;
    const int p0 = x.base + rb * ROWS / n.G, p1 = x.base + last / n.G;
    const int low1 = n.window ? p1 - n.window : -1;
    const AttnTiles tiles = at_tiles<32>(n, p0, p1);
    const int begin = part * a.tiles, end = begin + a.tiles < tiles.count ? begin + a.tiles : tiles.count;
    if (a.parts > 1 && part > 0 && begin >= tiles.count) return;
    const int keys = x.keys, D = n.D;

    auto key_of = [&](int i) { return 16 * (i >> 2) + 4 * quarter + (i & 3); };  // the lane's i-th key of a tile, as values
    auto score_of = [&](int i) { return key_of(col / ROWS * SC + i); };           // and as the scores that it works on
    // the pages of a tile's halves; the last key's in place of those behind it
    auto page_of = [&](int m, int half) -> int64_t {
        const int key = tiles.at(m) * 32 + 16 * half;
        return cache_page(s, b, (key < keys ? key : keys - 1) >> s.shift, hk);
    };
    auto load = [&](int m, const int64_t (&pages)[2], R& r) {
        const int key0 = tiles.at(m) * 32;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            r.bad[y] = pages[y] < 0;
            const int64_t page = pages[y] < 0 ? 0 : pages[y];
            const int at0 = (key0 + 16 * y) & (s.page - 1);
            const char* const kp = a.k + page;
            const char* const vp = a.v + page;
            // of a key, the lane's run of 8 KS elements
            const int at = at0 + col;
            if (FULL) {
                const int el = cache_unit(s, false, at, KS * quarter);
                __builtin_memcpy(r.k[y], kp + (KC == CACHE_F4 ? el / 2 : KC == CACHE_U8 ? el : 2 * el), 4 * R::KW * KS);
                if (KC == CACHE_F4) {
                    const char* const powers = kp + cache_power(s, false, at, 0);
                    const uint32_t first = ((const uint8_t*)powers)[KS * quarter >> 2];
                    const uint32_t last = DB == 3 ? ((const uint8_t*)powers)[(KS * quarter + KS - 1) >> 2] : first;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) r.kp[y][ks] = DB == 3 && (KS * quarter + ks) >> 2 != KS * quarter >> 2 ? last : first;
                }
            } else {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const int unit = KS * quarter + ks, el = cache_unit(s, false, at, 8 * unit < D ? unit : 0);
                    __builtin_memcpy(&r.k[y][ks * R::KW], kp + (KC == CACHE_F4 ? el / 2 : KC == CACHE_U8 ? el : 2 * el), 4 * R::KW);
                    if (KC == CACHE_F4) r.kp[y][ks] = ((const uint8_t*)kp)[cache_power(s, false, at, 8 * unit < D ? unit >> 2 : 0)];
                }
            }
            // of four tokens' values, the lane's block of eight elements (a half of it where NV is 4)
            const int unit = cache_lane_unit(DB, FULL, col, D), el = cache_unit(s, true, at0 + 4 * quarter, unit);
            __builtin_memcpy(r.v[y], vp + (KC == CACHE_F4 ? el / 2 : KC == CACHE_U8 ? el : 2 * el), 16 * R::KW);
            if (KC == CACHE_F4) __builtin_memcpy(&r.vp[y], vp + cache_power(s, true, at0 + 4 * quarter, unit >> 2), 4);
        }
    };
    R even, odd;
    int64_t pages[2] = {-1, -1};
    if (begin + w < end) {
        pages[0] = page_of(begin + w, 0);
        pages[1] = page_of(begin + w, 1);
        load(begin + w, pages, even);
        if (begin + w + 4 < end) {
            pages[0] = page_of(begin + w + 4, 0);
            pages[1] = page_of(begin + w + 4, 1);
        }
    }

    if (KC == CACHE_U8) {
        // low half: the value in bfloat16; high half: the same with zero for NaR (see AttnMarks)
        const uint32_t bits = bits_of_f32(posit_value(t, a.fc)) >> 16;
        const uint32_t e = bits | ((bits & 0x7F80u) == 0x7F80u ? 0u : bits << 16);
#pragma unroll
        for (int c = 0; c < 8; ++c) ((uint4*)smem)[t * 8 + c] = make_uint4(e, e, e, e);
        __syncthreads();
    }
    const uint32_t* const tab = smem + (lane & 31);

    float c = n.scale * 1.4426950408889634f;
    at_v8b q[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int d = 8 * (KS * quarter + ks);
        uint4 u = make_uint4(0, 0, 0, 0);
        if (live && col < ROWS && d < D) u = at_load8(a.q, (int64_t)(x.first + i) * a.ql + h * a.qh + d, 8, a.kq, a.fq);
        q[ks] = at_scaled(u, c);
    }
    c = at_scale(c);

    // eight elements of a key as bfloat16
    typedef __bf16 v2b __attribute__((ext_vector_type(2)));
    auto four = [&](uint32_t word, float scale, uint32_t (&o)[4]) {
        o[0] = __builtin_bit_cast(uint32_t, (v2b)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0));
        o[1] = __builtin_bit_cast(uint32_t, (v2b)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1));
        o[2] = __builtin_bit_cast(uint32_t, (v2b)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2));
        o[3] = __builtin_bit_cast(uint32_t, (v2b)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3));
    };
    auto entry = [&](uint32_t word, int i) -> uint32_t { return tab[((word >> (8 * i)) & 0xFFu) * 32]; };
    auto key_words = [&](const uint32_t* e, uint32_t power) -> uint4 {
        if constexpr (KC == CACHE_F4) {
            uint32_t o[4];
            four(e[0], f4_scale(power), o);
            return make_uint4(o[0], o[1], o[2], o[3]);
        } else if constexpr (KC == CACHE_U8) {
            auto two = [&](uint32_t word, int i) { return __builtin_amdgcn_perm(entry(word, i + 1), entry(word, i), 0x05040100u); };
            return make_uint4(two(e[0], 0), two(e[0], 2), two(e[1], 0), two(e[1], 2));
        } else {
            return make_uint4(e[0], e[1], e[2], e[3]);
        }
    };

    const float inf = f32_of_bits(0x7F800000u), nan = f32_of_bits(0x7FC00000u);
    float m = -inf, l = 0.f;
    at_v4f o[NV];
#pragma unroll
    for (int y = 0; y < NV; ++y) o[y] = at_v4f{0.f, 0.f, 0.f, 0.f};
    uint32_t flagged = 0;
    auto step = [&](int tile, const R& cur, R& next) {
        if (tile + 4 < end) {
            load(tile + 4, pages, next);
            if (tile + 8 < end) {
                pages[0] = page_of(tile + 8, 0);
                pages[1] = page_of(tile + 8, 1);
            }
        }
        const int key0 = tiles.at(tile) * 32;
        float all[8];  // of keys key_of(0 .. 7)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            at_v4f acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                uint4 u = key_words(&cur.k[y][ks * R::KW], KC == CACHE_F4 ? cur.kp[y][ks] : 0u);
                if (!FULL) u = 8 * (KS * quarter + ks) < D ? u : make_uint4(0, 0, 0, 0);
                acc = at_mfma16(at_frag(u), q[ks], acc);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) all[4 * y + r] = acc[r];
        }
        // pages that are none; blocks of NaN, a block of a key to a lane
        if (cur.bad[0] || cur.bad[1]) {
#pragma unroll
            for (int r = 0; r < 8; ++r) all[r] = cur.bad[r >> 2] ? nan : all[r];
        }
        if (KC == CACHE_F4) {
            bool gone[2] = {false, false};
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) gone[y] |= cur.kp[y][ks] == 255u;
            if (__any(gone[0] || gone[1])) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint64_t lanes = __ballot(gone[y]);
                    const uint32_t keys16 = (uint32_t)(lanes | lanes >> 16 | lanes >> 32 | lanes >> 48);
#pragma unroll
                    for (int r = 0; r < 4; ++r) all[4 * y + r] = (keys16 >> (4 * quarter + r)) & 1u ? nan : all[4 * y + r];
                }
            }
        }
        float sc[SC];  // of keys score_of(0 ..)
#pragma unroll
        for (int r = 0; r < SC; ++r) {
            sc[r] = all[r];
            if (ROWS == 8) sc[r] = spread<8, 0xC>(sc[r], all[(SC + r) & 7]);
            if (ROWS == 4) sc[r] = spread<12, 0x8>(spread<8, 0x4>(spread<4, 0x2>(sc[r], all[(2 + r) & 7]), all[(4 + r) & 7]), all[(6 + r) & 7]);
        }
        if (!(key0 + 31 <= p0 && (key0 > low1 || key0 + 31 < n.sinks))) {
#pragma unroll
            for (int r = 0; r < SC; ++r) sc[r] = at_sees(n, p, low, key0 + score_of(r)) ? sc[r] : -inf;
        }
        float mx = sc[0];
#pragma unroll
        for (int r = 1; r < SC; ++r) mx = fmaxf(mx, sc[r]);
        if (ROWS <= 8) mx = fmaxf(mx, turned<8>(mx));
        if (ROWS <= 4) mx = fmaxf(mx, turned<4>(mx));
        mx = at_max_halves(max_rows(mx)) * c;
        if (__any(mx > m + 8.f)) {
            const float m1 = fmaxf(m, mx), f = m1 == -inf ? 1.f : __builtin_amdgcn_exp2f(m - m1);
            m = m1;
            l *= f;
#pragma unroll
            for (int y = 0; y < NV; ++y) o[y] *= f;
        }
        const float mr = m == -inf ? 0.f : m;
#pragma unroll
        for (int r = 0; r < SC; ++r) {
            sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], c, -mr));
            l += sc[r];
        }
        // the probabilities in two parts, back to the lanes whose columns they are
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int r = 0; r < SC / 2; ++r) {
            v2b h = {(__bf16)sc[2 * r], (__bf16)sc[2 * r + 1]};
            hi[r] = __builtin_bit_cast(uint32_t, h);
            v2b g = {(__bf16)(sc[2 * r] - f32_of_bits(hi[r] << 16)), (__bf16)(sc[2 * r + 1] - f32_of_bits(hi[r] & 0xFFFF0000u))};
            lo[r] = __builtin_bit_cast(uint32_t, g);
        }
        if (ROWS == 8) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                hi[2 + r] = from_above<8>(hi[r]);
                lo[2 + r] = from_above<8>(lo[r]);
            }
        }
        if (ROWS == 4) {
            hi[1] = from_above<4>(hi[0]);
            hi[2] = from_above<8>(hi[0]);
            hi[3] = from_above<12>(hi[0]);
            lo[1] = from_above<4>(lo[0]);
            lo[2] = from_above<8>(lo[0]);
            lo[3] = from_above<12>(lo[0]);
        }
        const at_v8b ph = at_frag(make_uint4(hi[0], hi[1], hi[2], hi[3])), pl = at_frag(make_uint4(lo[0], lo[1], lo[2], lo[3]));

        // what lies behind the last key is anything: zeros
        uint32_t v[2][4 * R::KW], vp[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
#pragma unroll
            for (int e = 0; e < 4 * R::KW; ++e) v[y][e] = cur.v[y][e];
            if (KC == CACHE_F4) vp[y] = cur.vp[y];
        }
        if (key0 + 31 >= keys) {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool in = key0 + key_of(4 * y + e) < keys;
#pragma unroll
                    for (int z = 0; z < R::KW; ++z) v[y][e * R::KW + z] = in ? v[y][e * R::KW + z] : 0u;
                    if (KC == CACHE_F4) vp[y] = in ? vp[y] : (vp[y] & ~(0xFFu << (8 * e))) | 127u << (8 * e);
                }
        }
        // NaR, NaN and infinities: zeros, and looked up at the end
        uint32_t special = 0;
        if (KC == CACHE_F4) {
#pragma unroll
            for (int y = 0; y < 2; ++y) special |= (~vp[y] - 0x01010101u) & vp[y] & 0x80808080u;
        } else if (KC == CACHE_U8) {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t z = v[y][e] ^ 0x80808080u;
                    special |= (z - 0x01010101u) & ~z & 0x80808080u;
                }
        } else {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int e = 0; e < 16; ++e) special |= at_odd(v[y][e]) ? 1u : 0u;
        }
        flagged |= special;
        if (KC != CACHE_U8 && __any(special != 0)) {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (KC == CACHE_F4) {
                        const bool gone = ((vp[y] >> (8 * e)) & 0xFFu) == 255u;
                        v[y][e] = gone ? 0u : v[y][e];
                        vp[y] = gone ? vp[y] ^ 128u << (8 * e) : vp[y];
                    } else {
#pragma unroll
                        for (int z = 0; z < 4; ++z) {
                            uint32_t u = v[y][(4 * e + z) % (4 * R::KW)];
                            if ((u & 0x7F80u) == 0x7F80u) u &= 0xFFFF0000u;
                            if ((u & 0x7F800000u) == 0x7F800000u) u &= 0xFFFFu;
                            v[y][(4 * e + z) % (4 * R::KW)] = u;
                        }
                    }
                }
        }
        // the NV elements of each of the lane's eight keys; two keys' to a word
        const bool high = NV == 4 && (col & 1);
        if constexpr (KC == CACHE_F4) {
            uint32_t d[8][4];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float scale = f4_scale((vp[e / 4] >> (8 * (e & 3))) & 0xFFu);
                const uint32_t word = high ? v[e / 4][e & 3] >> 16 : v[e / 4][e & 3];
                d[e][0] = __builtin_bit_cast(uint32_t, (v2b)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0));
                d[e][1] = __builtin_bit_cast(uint32_t, (v2b)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1));
                if (NV == 8) {
                    d[e][2] = __builtin_bit_cast(uint32_t, (v2b)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2));
                    d[e][3] = __builtin_bit_cast(uint32_t, (v2b)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3));
                }
            }
#pragma unroll
            for (int y = 0; y < NV; ++y) {
                const uint32_t sel = y & 1 ? 0x07060302u : 0x05040100u;
                const at_v8b f = at_frag(make_uint4(__builtin_amdgcn_perm(d[1][y / 2], d[0][y / 2], sel), __builtin_amdgcn_perm(d[3][y / 2], d[2][y / 2], sel),
                                                    __builtin_amdgcn_perm(d[5][y / 2], d[4][y / 2], sel), __builtin_amdgcn_perm(d[7][y / 2], d[6][y / 2], sel)));
                o[y] = at_mfma16(f, ph, o[y]);
                o[y] = at_mfma16(f, pl, o[y]);
            }
        } else {
            constexpr int KW = R::KW;
            // words of the lane's NV elements
            constexpr int W = NV * KW / 8;
            uint32_t d[8][W];
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int z = 0; z < W; ++z) {
                    const uint32_t first = v[e / 4][(e & 3) * KW + z], second = v[e / 4][(e & 3) * KW + (z + KW / 2) % KW];
                    d[e][z] = NV == 4 && high ? second : first;
                }
#pragma unroll
            for (int y = 0; y < NV; ++y) {
                uint32_t u[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (KC == CACHE_U8) u[e] = __builtin_amdgcn_perm(entry(d[2 * e + 1][y / 4 % W], y & 3), entry(d[2 * e][y / 4 % W], y & 3), 0x07060302u);
                    else u[e] = __builtin_amdgcn_perm(d[2 * e + 1][y / 2 % W], d[2 * e][y / 2 % W], y & 1 ? 0x07060302u : 0x05040100u);
                }
                const at_v8b f = at_frag(make_uint4(u[0], u[1], u[2], u[3]));
                o[y] = at_mfma16(f, ph, o[y]);
                o[y] = at_mfma16(f, pl, o[y]);
            }
        }
    };
    for (int tile = begin + w; tile < end; tile += 8) {
        step(tile, even, odd);
        if (tile + 4 < end) step(tile + 4, odd, even);
    }
    if (ROWS <= 8) l += turned<8>(l);
    if (ROWS <= 4) l += turned<4>(l);
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (__any(flagged != 0)) {
        // the wave's tiles once more, an element of a value to a lane
        AttnMarks<DB> marks = {};
        for (int tile = begin + w; tile < end; tile += 4) {
            const int64_t at[2] = {page_of(tile, 0), page_of(tile, 1)};
#pragma unroll 4
            for (int r = 0; r < 32; ++r) {
                const int key = tiles.at(tile) * 32 + r;
                const char* const from = a.v + (at[r >> 4] < 0 ? 0 : at[r >> 4]);
                uint32_t mk[3][4] = {};
#pragma unroll
                for (int y = 0; y < (DB + 1) / 2; ++y) {
                    const int d = 64 * y + lane;
                    float v = 0.f;
                    if (d < D && key < keys) {
                        const int slot = key & (s.page - 1), el = cache_unit(s, true, slot, d >> 3) + (d & 7);
                        if (KC == CACHE_F4) v = ((const uint8_t*)from)[cache_power(s, true, slot, d >> 5)] == 255u ? nan : 0.f;
                        else if (KC == CACHE_U8) v = posit_value(((const uint8_t*)from)[el], a.fc);
                        else v = f32_of_bits((uint32_t)((const uint16_t*)from)[el] << 16);
                    }
                    const uint64_t bits[3] = {__ballot(v == inf), __ballot(v == -inf), __ballot(v != v)};
#pragma unroll
                    for (int z = 0; z < 3; ++z) {
                        mk[z][2 * y] = (uint32_t)bits[z];
                        mk[z][2 * y + 1] = (uint32_t)(bits[z] >> 32);
                    }
                }
                marks.add(mk[0], mk[1], mk[2], at_sees(n, p, low, key));
            }
        }
        // the lane's elements NV (4 quarter + r) + y lie in one word
        const int word = NV * quarter / 8, from = NV * 4 * quarter & 31;
        uint32_t mp = 0, mn = 0, mq = 0;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            mp = word == d ? marks.pos[d] : mp;
            mn = word == d ? marks.neg[d] : mn;
            mq = word == d ? marks.nan[d] : mq;
        }
#pragma unroll
        for (int y = 0; y < NV; ++y)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[y][r] = at_marked(o[y][r], mp, mn, mq, from + NV * r + y);
    }

    // join the waves: a common reference, then through LDS, [wave][block][element row][column]
    if (quarter == 0 && col < ROWS) {
        wm[w][col] = m;
        wl[w][col] = l;
    }
    __syncthreads();
    const int cr = col % ROWS;
    const float top = fmaxf(fmaxf(wm[0][cr], wm[1][cr]), fmaxf(wm[2][cr], wm[3][cr]));
    const float f = m == -inf ? 1.f : __builtin_amdgcn_exp2f(m - top);
    float* const red = (float*)smem;
#pragma unroll
    for (int y = 0; y < NV; ++y)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float u = o[y][r];
            red[((w * NV + y) * 16 + 4 * quarter + r) * 16 + col] = u - u == 0.f ? u * f : u;  // an infinity stays one
        }
    __syncthreads();
    // NV neighbouring elements of a row to a thread
    const int rr = t >> 4, rho = t & 15, gr = rb * ROWS + rr, d = NV * rho;
    if (rr >= ROWS || gr >= x.rows) return;
    float out[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int y = 0; y < NV; ++y)
#pragma unroll
        for (int z = 0; z < 4; ++z) out[y] += red[((z * NV + y) * 16 + rho) * 16 + rr];
    float mm = -inf, sum = 0.f;
#pragma unroll
    for (int z = 0; z < 4; ++z) mm = fmaxf(mm, wm[z][rr]);
#pragma unroll
    for (int z = 0; z < 4; ++z) sum += wm[z][rr] == -inf ? wl[z][rr] : wl[z][rr] * __builtin_amdgcn_exp2f(wm[z][rr] - mm);
    if (a.parts > 1 && tiles.count > a.tiles) {
        float* const at = a.part + ((((int64_t)b * s.HKV + hk) * a.blocks + rb) * a.parts + part) * (ROWS * (D + 2));
        if (rho == 0) {
            at[rr] = mm;
            at[ROWS + rr] = sum;
        }
#pragma unroll
        for (int y = 0; y < NV; ++y)
            if (d + y < D) at[2 * ROWS + rr * D + d + y] = out[y];
        return;
    }
    const int gi = gr / n.G, gh = hk * n.G + (gr - gi * n.G);
    const int64_t to = (int64_t)(x.first + gi) * (s.HKV * n.G) + gh;
    if (a.lse && rho == 0) a.lse[to] = sum == 0.f ? -inf : mm * 0.6931471805599453f + logf(sum);
    const float up = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int y = 0; y < 8; ++y) out[y] *= up;
    at_store8(a.o, to * D + d, D - d < NV ? D - d : NV, a.ko, a.fo, out);
}

// Latency: the parts' maxima, then their rows with all loads in flight; 1 x 60000, 94 parts: 5 us.
// Parts of a row joined, one row to a workgroup, an element to a thread of each four, which take the parts in turn; rows whose keys are in one part are done.
__global__ __launch_bounds__(512) void attn_paged_join_kernel(AttnPaged a) {
    __shared__ float weight[AT_MOST_PARTS];
    __shared__ float wave_max_of[4], wave_sum_of[4], sums[4][128];
    const AttnShape& n = a.n;
    const int row = blockIdx.x, hk = blockIdx.y, b = blockIdx.z, t = threadIdx.x, rb = row / a.rows, rr = row - rb * a.rows, D = n.D;
    const PagedRows x(a, b);
    if (row >= x.rows) return;
    const int i = row / n.G, h = hk * n.G + (row - i * n.G);
    const int last = rb * a.rows + a.rows - 1 < x.rows ? rb * a.rows + a.rows - 1 : x.rows - 1;
    const int count = at_tiles<32>(n, x.base + rb * a.rows / n.G, x.base + last / n.G).count;
    if (count <= a.tiles) return;
    const int parts = (count + a.tiles - 1) / a.tiles;
    const int64_t step = a.rows * (D + 2);
    const float* const at = a.part + ((((int64_t)b * a.s.HKV + hk) * a.blocks + rb) * a.parts) * step;
    const float inf = f32_of_bits(0x7F800000u);
    // a part to a thread of the first four waves
    const bool mine = t < parts;
    const float m0 = mine ? at[t * step + rr] : -inf, s0 = mine ? at[t * step + a.rows + rr] : 0.f;
    // the outputs are on their way meanwhile
    const int e = t & 127, g = t >> 7;
    const float* const from = at + 2 * a.rows + rr * D + (e < D ? e : 0);
    float v[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) v[y] = from[(g + 4 * y < parts ? g + 4 * y : 0) * step];
    float m = wave_max(m0);
    if ((t & 63) == 0 && t < 256) wave_max_of[t >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(wave_max_of[0], wave_max_of[1]), fmaxf(wave_max_of[2], wave_max_of[3]));
    const float f = m0 == -inf ? 1.f : __builtin_amdgcn_exp2f(m0 - m);  // a part without keys: zeros, or NaN
    if (t < AT_MOST_PARTS) weight[t] = f;
    float l = wave_sum(s0 * f);
    if ((t & 63) == 0 && t < 256) wave_sum_of[t >> 6] = l;
    __syncthreads();
    l = (wave_sum_of[0] + wave_sum_of[1]) + (wave_sum_of[2] + wave_sum_of[3]);
    const int64_t to = (int64_t)(x.first + i) * (a.s.HKV * n.G) + h;
    if (a.lse && t == 0) a.lse[to] = l == 0.f ? -inf : m * 0.6931471805599453f + logf(l);
    float o = 0.f;
    for (int p = g; p < parts; p += 32) {
#pragma unroll
        for (int y = 0; y < 8; ++y)
            if (p + 4 * y < parts) o += v[y] - v[y] == 0.f ? v[y] * weight[p + 4 * y] : v[y];
        if (p + 32 < parts)
#pragma unroll
            for (int y = 0; y < 8; ++y) v[y] = from[(p + 32 + 4 * y < parts ? p + 32 + 4 * y : 0) * step];
    }
    sums[g][e] = o;
    __syncthreads();
    if (t >= D) return;
    o = (sums[0][t] + sums[1][t]) + (sums[2][t] + sums[3][t]);
    o = l == 0.f ? 0.f : o / l;
    store_value(a.o, to * D + t, a.ko, a.fo, o);
}

// A cache without pages, which has nothing to read: every token lies in a page that is none, so a row that sees one is NaN.  A new row to a workgroup.
__global__ __launch_bounds__(256) void attn_paged_none_kernel(AttnPaged a) {
    const int i = blockIdx.x, b = blockIdx.y;
    const PagedRows x(a, b);
    if (i >= x.count) return;
    const bool sees = x.base + i >= 0;  // itself
    const int heads = a.n.HKV * a.n.G;
    const int64_t row = x.first + i;
    for (int64_t e = threadIdx.x; e < (int64_t)heads * a.n.D; e += 256) store_value(a.o, row * heads * a.n.D + e, a.ko, a.fo, f32_of_bits(sees ? 0x7FC00000u : 0u));
    if (a.lse)
        for (int h = threadIdx.x; h < heads; h += 256) a.lse[row * heads + h] = f32_of_bits(sees ? 0x7FC00000u : 0xFF800000u);
}

}  // namespace pnn
