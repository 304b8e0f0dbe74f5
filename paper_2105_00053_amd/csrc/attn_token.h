// Attention of few queries on long caches: single tokens of a batch, or the last few of a prompt.
//
// A workgroup takes up to 32 rows (positions and heads of a group) and a part of the keys that they see; its four waves take tiles of 32
// keys in turn, each with a running maximum, sum and result of its own, joined in LDS at the end and, where a sequence was split
// over workgroups, by a second kernel.  Bound by memory: an element of the cache is read once and used for every head of the group, so it is decoded
// where it is used.  8-bit posits go through a table in LDS that every bank has a copy of (32 KB; look-ups without conflicts): two vector
// operations and a half an element, where the field decoder takes 14.
// The reduction order of the second product is free, so a lane takes four neighbouring elements of a head (one load) of 16 keys as
// they lie in memory: result row rho of block x is element 4 rho + x.
#pragma once

#include "attn_prompt.h"

namespace pnn {

struct AttnToken {
    AttnShape s;
    const void *q, *k, *v;
    int64_t qb, ql, qh, kb, kl, kh, vb, vl, vh;
    int kq;
    ElemFmt fq, fkv;
    void *o, *copy;
    float* lse;
    int ko, kc;
    ElemFmt fo, fc;
    int tiles;    // of a part
    int parts;    // workgroups that a row block's keys are split over
    float* part;  // for more than one: [row block][part][m: 32][l: 32][32][D]
};

// A tile's keys and values as they lie in memory, in words: 8 elements of a key at a time, 4 of a value.
template <int K, int KS>
struct AttnRaw {
    static constexpr int B = sizeof(typename Raw<K>::T);
    uint32_t k[KS][2 * B], v[16][B];
};

// N elements (4 or 8) from `src`, zeros in place of those beyond `left`
template <class T, int N>
__device__ __forceinline__ void at_words(const T* src, int left, uint32_t (&o)[N * sizeof(T) / 4]) {
    if (left >= N) {
        __builtin_memcpy(o, src, N * sizeof(T));
        return;
    }
    constexpr int PER = 4 / sizeof(T);
#pragma unroll
    for (int i = 0; i < N / PER; ++i) {
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (i * PER + j < left) w |= (uint32_t)src[i * PER + j] << (8 * sizeof(T) * j);
        o[i] = w;
    }
}

// Results of a row: divided by the sum, rounded to the output and its copy.
template <class A>
__device__ __forceinline__ void at_store(const A& a, int64_t at, int d, float v) {
    store_value(a.o, at + d, a.ko, a.fo, v);
    if (a.copy) store_value(a.copy, at + d, a.kc, a.fc, v);
}

template <int K, int DB, bool TWO>
__global__ __launch_bounds__(256, 2) void attn_token_kernel(AttnToken a) {
    constexpr int KS = 2 * DB;
    __shared__ uint32_t smem[8192];  // the table, then what the waves join through
    __shared__ float wm[4][32], wl[4][32];
    const AttnShape& s = a.s;
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), half = lane >> 5, col = lane & 31;
    const int hk = blockIdx.y, b = blockIdx.z;
    const int rb = blockIdx.x / (unsigned)a.parts, part = blockIdx.x - rb * a.parts;
    const int base = at_keys(s, b) - s.LQ;
    const int row = rb * 32 + col, last = (rb * 32 + 31 < s.rows ? rb * 32 + 31 : s.rows - 1);
    const int i = row / s.G, h = hk * s.G + (row - i * s.G);
    const bool live = row < s.rows;
    const int p = live ? base + i : -1, low = s.window ? p - s.window : -1;
    const int p0 = base + rb * 32 / s.G, p1 = base + last / s.G;
    const int low1 = s.window ? p1 - s.window : -1;
    const AttnTiles tiles = at_tiles<32>(s, p0, p1);
    const int begin = part * a.tiles, end = begin + a.tiles < tiles.count ? begin + a.tiles : tiles.count;

    if (K == KIND_POSIT_U8) {
        // low half: the value in bfloat16; high half: the same with zero for NaR (see AttnMarks)
        const uint32_t bits = bits_of_f32(posit_value(t, a.fkv)) >> 16;
        const uint32_t e = bits | ((bits & 0x7F80u) == 0x7F80u ? 0u : bits << 16);
#pragma unroll
        for (int c = 0; c < 8; ++c) ((uint4*)smem)[t * 8 + c] = make_uint4(e, e, e, e);
        __syncthreads();
    }
    const uint32_t* const tab = smem + col;

    float c = s.scale * 1.4426950408889634f;
    at_v8b q[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int d = ks * 16 + 8 * half;
        uint4 u = make_uint4(0, 0, 0, 0);
        if (live && d < s.D) u = at_load8(a.q, b * a.qb + i * a.ql + h * a.qh + d, s.D - d, a.kq, a.fq);
        q[ks] = at_scaled(u, c);
    }
    c = at_scale(c);

    typedef typename Raw<K>::T T;
    const T* const ksrc = (const T*)a.k + b * a.kb + hk * a.kh;
    const T* const vsrc = (const T*)a.v + b * a.vb + hk * a.vh;
    const int keys = base + s.LQ;
    auto load_keys = [&](int n, AttnRaw<K, KS>& r) {
        const int key0 = tiles.at(n) * 32;
        {
            const int key = key0 + col;
            const T* src = ksrc + (int64_t)(key < keys ? key : keys - 1) * a.kl;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) at_words<T, 8>(src + ks * 16 + 8 * half, s.D - (ks * 16 + 8 * half), r.k[ks]);
        }
    };
    auto load_values = [&](int n, AttnRaw<K, KS>& r) {
        const int key0 = tiles.at(n) * 32;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int key = key0 + (e >> 3) * 16 + at_row(e & 7, half);
            at_words<T, 4>(vsrc + (int64_t)(key < keys ? key : keys - 1) * a.vl + 4 * col, s.D - 4 * col, r.v[e]);
        }
    };
    // element i of a row of words, its bfloat16 in the low half; two of them
    constexpr int PER = 4 / sizeof(T), BITS = 8 * sizeof(T);
    auto entry = [&](const uint32_t* words, int i) -> uint32_t {
        const uint32_t raw = (words[i / PER] >> (BITS * (i % PER))) & ((1u << BITS) - 1u);
        if (K == KIND_POSIT_U8) return tab[raw * 32];
        return K == KIND_BF16 ? raw : bits_of_f32(posit_value(raw, a.fkv)) >> 16;
    };
    auto pair = [&](const uint32_t* w0, int i0, const uint32_t* w1, int i1, bool value) -> uint32_t {
        uint32_t e0 = entry(w0, i0), e1 = entry(w1, i1);
        if (K == KIND_POSIT_U8) return __builtin_amdgcn_perm(e1, e0, value ? 0x07060302u : 0x05040100u);
        if (value) {
            e0 = (e0 & 0x7F80u) == 0x7F80u ? 0u : e0;
            e1 = (e1 & 0x7F80u) == 0x7F80u ? 0u : e1;
        }
        return __builtin_amdgcn_perm(e1, e0, 0x05040100u);
    };
    // nonzero where a word of values holds a NaR, a NaN or an infinity
    auto odd = [&](uint32_t word) -> uint32_t {
        if (K == KIND_POSIT_U8) {
            const uint32_t x = word ^ 0x80808080u;
            return (x - 0x01010101u) & ~x & 0x80808080u;
        }
        const uint32_t m = K == KIND_BF16 ? 0x7F80u : (1u << a.fkv.n) - 1u, want = K == KIND_BF16 ? 0x7F80u : 1u << (a.fkv.n - 1);
        return (word & m) == want || ((word >> 16) & m) == want;
    };

    const float inf = f32_of_bits(0x7F800000u);
    float m = -inf, l = 0.f;
    at_v16f o[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) o[x] = at_zero();
    uint32_t flagged = 0;
    AttnRaw<K, KS> raw;
    // the next tile is on its way while one is worked on; of 16-bit elements only its keys, for which there are registers
    constexpr bool AHEAD = sizeof(T) == 1;
    if (begin + w < end) {
        load_keys(begin + w, raw);
        if (AHEAD) load_values(begin + w, raw);
    }
    for (int n = begin + w; n < end; n += 4) {
        if (!AHEAD) load_values(n, raw);
        const AttnRaw<K, KS> cur = raw;
        if (n + 4 < end) {
            load_keys(n + 4, raw);
            if (AHEAD) load_values(n + 4, raw);
        }
        const int key0 = tiles.at(n) * 32;
        at_v16f sc = at_zero();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const uint32_t* e = cur.k[ks];
            sc = at_mfma(at_frag(make_uint4(pair(e, 0, e, 1, false), pair(e, 2, e, 3, false), pair(e, 4, e, 5, false), pair(e, 6, e, 7, false))), q[ks], sc);
        }
        if (!(key0 + 31 <= p0 && (key0 > low1 || key0 + 31 < s.sinks))) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[r] = at_sees(s, p, low, key0 + at_row(r, half)) ? sc[r] : -inf;
        }
        float mx = sc[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[r]);
        mx = at_max_halves(mx) * c;
        if (__any(mx > m + 8.f)) {
            const float m1 = fmaxf(m, mx), f = m1 == -inf ? 1.f : __builtin_amdgcn_exp2f(m - m1);
            m = m1;
            l *= f;
#pragma unroll
            for (int x = 0; x < 4; ++x) o[x] *= f;
        }
        const float mr = m == -inf ? 0.f : m;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], c, -mr));
            l += sc[r];
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
            for (int x = 0; x < AttnRaw<K, KS>::B; ++x) flagged |= odd(cur.v[e][x]);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const at_v8b ph = at_round(sc, 8 * y);
            at_v8b pl;
            if (TWO) pl = at_rest(sc, 8 * y, ph);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                uint32_t u[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = pair(cur.v[8 * y + 2 * e], x, cur.v[8 * y + 2 * e + 1], x, true);
                const at_v8b v = at_frag(make_uint4(u[0], u[1], u[2], u[3]));
                o[x] = at_mfma(v, ph, o[x]);
                if (TWO) o[x] = at_mfma(v, pl, o[x]);
            }
        }
    }
    l += __shfl_xor(l, 32, 64);
    if (__any(flagged != 0)) {
        AttnMarks marks = {};
        for (int n = begin + w; n < end; n += 4)
            for (int j = tiles.at(n) * 32; j < tiles.at(n) * 32 + 32; ++j)
                if (at_sees(s, p, low, j))
#pragma unroll 1
                    for (int e = 0; e < 64; ++e) {
                        const int d = 4 * at_row(e & 15, half) + (e >> 4);
                        if (d < s.D) marks.add(e, value_of<K>(vsrc[j * a.vl + d], a.fkv));
                    }
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[x][r] = marks.apply(16 * x + r, o[x][r]);
    }

    // join the waves: a common reference, then block by block through LDS
    if (half == 0) {
        wm[w][col] = m;
        wl[w][col] = l;
    }
    __syncthreads();
    const float top = fmaxf(fmaxf(wm[0][col], wm[1][col]), fmaxf(wm[2][col], wm[3][col]));
    const float f = m == -inf ? 1.f : __builtin_amdgcn_exp2f(m - top);
    float* const red = (float*)smem;
    float out[4][4];  // [k][x]: element 4 (t % 32) + x of row t / 32 + 8 k
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        if (x > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float v = o[x][r];
            red[(w * 32 + at_row(r, half)) * 33 + col] = v - v == 0.f ? v * f : v;  // an infinity stays one
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float v = 0.f;
#pragma unroll
            for (int y = 0; y < 4; ++y) v += red[(y * 32 + (t & 31)) * 33 + (t >> 5) + 8 * k];
            out[k][x] = v;
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int rr = (t >> 5) + 8 * k, gr = rb * 32 + rr, d = 4 * (t & 31);
        if (gr >= s.rows) continue;
        float mm = -inf, sum = 0.f;
#pragma unroll
        for (int y = 0; y < 4; ++y) mm = fmaxf(mm, wm[y][rr]);
#pragma unroll
        for (int y = 0; y < 4; ++y) sum += wm[y][rr] == -inf ? wl[y][rr] : wl[y][rr] * __builtin_amdgcn_exp2f(wm[y][rr] - mm);
        if (a.parts > 1) {
            float* const at = a.part + ((((int64_t)b * s.HKV + hk) * (gridDim.x / a.parts) + rb) * a.parts + part) * (32 * (s.D + 2));
            if ((t & 31) == 0) {
                at[rr] = mm;
                at[32 + rr] = sum;
            }
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (d + x < s.D) at[64 + rr * s.D + d + x] = out[k][x];
            continue;
        }
        const int gi = gr / s.G, gh = hk * s.G + (gr - gi * s.G);
        if (a.lse && (t & 31) == 0) a.lse[((int64_t)b * s.HKV * s.G + gh) * s.LQ + gi] = sum == 0.f ? -inf : mm * 0.6931471805599453f + logf(sum);
        const float up = sum == 0.f ? 0.f : 1.f / sum;
        const int64_t at = (((int64_t)b * s.LQ + gi) * (s.HKV * s.G) + gh) * s.D;
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (d + x < s.D) at_store(a, at, d + x, out[k][x] * up);
    }
}

// Parts of a row joined, one row to a workgroup and an element to a thread.
__global__ __launch_bounds__(128) void attn_join_kernel(AttnToken a) {
    const AttnShape& s = a.s;
    const int row = blockIdx.x, hk = blockIdx.y, b = blockIdx.z, d = threadIdx.x, rr = row & 31;
    const int i = row / s.G, h = hk * s.G + (row - i * s.G), blocks = (s.rows + 31) / 32;
    const int64_t step = 32 * (s.D + 2);
    const float* const at = a.part + (((int64_t)b * s.HKV + hk) * blocks + (row >> 5)) * a.parts * step;
    const float inf = f32_of_bits(0x7F800000u);
    float m = -inf, l = 0.f, o = 0.f;
    for (int n = 0; n < a.parts; ++n) m = fmaxf(m, at[n * step + rr]);
    for (int n = 0; n < a.parts; ++n) {
        const float mn = at[n * step + rr], ln = at[n * step + 32 + rr];
        const float f = mn == -inf ? 1.f : __builtin_amdgcn_exp2f(mn - m);
        l += ln * f;
        if (d < s.D) {
            const float v = at[n * step + 64 + rr * s.D + d];
            o += v - v == 0.f ? v * f : v;
        }
    }
    if (a.lse && d == 0) a.lse[((int64_t)b * s.HKV * s.G + h) * s.LQ + i] = l == 0.f ? -inf : m * 0.6931471805599453f + logf(l);
    if (d < s.D) at_store(a, (((int64_t)b * s.LQ + i) * (s.HKV * s.G) + h) * s.D, d, l == 0.f ? 0.f : o / l);
}

}  // namespace pnn
