// Attention of few queries on long caches: single tokens of a batch, or the last few of a prompt.
//
// A workgroup takes up to 16 rows (positions and heads of a group) and a part of the keys that they see; its four waves take tiles of 32
// keys in turn, each with a running maximum, sum and result of its own, joined in LDS at the end and, where a sequence was split
// over workgroups, by a second kernel.  Bound by memory in principle: an element of the cache is read once and used for every head of the group, so it is decoded
// where it is used.  8-bit posits go through a table in LDS that every bank has a copy of (32 KB; look-ups without conflicts): two vector
// operations and a half an element, where the field decoder takes 12.
//
// 48 sequences of up to 8192 keys, window 4096, 8 heads of 128 for 32 of queries, 8-bit posits: 97 to 101 us for 335 MB, 3.4 TB/s (vector unit 44 % of the cycles, LDS 21,
// 1.5 waves on a SIMD: latencies of loads and look-ups); 16 of 4096 in bfloat16 48, 5.6 TB/s; in 12-bit posits by the field decoder 120, 2.2 TB/s (vector unit 72 %).  One
// sequence of 8192: 21, 3 of 300: 8.
//
// v_mfma_f32_16x16x32_bf16 (a group of heads rarely has more than 16; on the 32 x 32 form results and q took twice the registers): lane l
// holds, for A, row l % 16 and the 8 reduction indices from 8 (l / 16); for B, column l % 16 and the same; result register r is row 4 (l / 16) + r,
// column l % 16.  S^T = K Q^T (two blocks of 16 keys), then O^T += V^T P^T: a lane's eight probabilities are the keys 16 (i / 4) + 4 (l / 16) + i % 4, which
// is the order that its values are loaded in.  The rows of O^T are in any order too: a lane loads NV neighbouring elements of a value (one
// load) and gives one to each of NV blocks, so row rho of block x is element NV rho + x.
#pragma once

#include "attn_prompt.h"

namespace pnn {

typedef float at_v4f __attribute__((ext_vector_type(4)));
__device__ __forceinline__ at_v4f at_mfma16(at_v8b a, at_v8b b, at_v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

constexpr int AT_TOKEN_ROWS = 16;
constexpr int AT_MOST_PARTS = 256;  // workgroups to a row block's keys, what the second kernel holds weights of

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
    float* part;  // for more than one: [row block][part][m: 16][l: 16][16][D]
};

// A tile's keys and values as they lie in memory, in words: 8 elements of a key at a time, NV of a value.
template <int K, int KS, int NV>
struct AttnRaw {
    static constexpr int B = sizeof(typename Raw<K>::T);
    uint32_t k[2][KS][2 * B], v[8][NV * B / 4];
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

// WHOLE: heads of a multiple of 8 elements, so that a vector lies inside one or outside; those outside are read from the head's start and, of keys,
// taken as zero (of values they go to elements that do not exist).
template <int K, int DB, bool WHOLE>
__global__ __launch_bounds__(256, sizeof(typename Raw<K>::T) == 1 ? 3 : 2) void attn_token_kernel(AttnToken a) {
    constexpr int KS = DB, NV = DB <= 2 ? 4 : 8;
    __shared__ uint32_t smem[8192];  // the table, then what the waves join through
    __shared__ float wm[4][16], wl[4][16];
    const AttnShape& s = a.s;
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), quarter = lane >> 4, col = lane & 15;
    const int hk = blockIdx.y, b = blockIdx.z;
    const int rb = blockIdx.x / (unsigned)a.parts, part = blockIdx.x - rb * a.parts;
    const int base = at_keys(s, b) - s.LQ;
    const int row = rb * 16 + col, last = (rb * 16 + 15 < s.rows ? rb * 16 + 15 : s.rows - 1);
    const int i = row / s.G, h = hk * s.G + (row - i * s.G);
    const bool live = row < s.rows;
    const int p = live ? base + i : -1, low = s.window ? p - s.window : -1;
    const int p0 = base + rb * 16 / s.G, p1 = base + last / s.G;
    const int low1 = s.window ? p1 - s.window : -1;
    const AttnTiles tiles = at_tiles<32>(s, p0, p1);
    const int begin = part * a.tiles, end = begin + a.tiles < tiles.count ? begin + a.tiles : tiles.count;

    typedef typename Raw<K>::T T;
    typedef AttnRaw<K, KS, NV> R;
    const T* const ksrc = (const T*)a.k + b * a.kb + hk * a.kh;
    const T* const vsrc = (const T*)a.v + b * a.vb + hk * a.vh;
    const int keys = base + s.LQ;
    auto key_of = [&](int i) { return 16 * (i >> 2) + 4 * quarter + (i & 3); };  // the lane's i-th key of a tile, as scores and as values
    auto load_keys = [&](int n, R& r) {
        const int key0 = tiles.at(n) * 32;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int key = key0 + 16 * x + col;
            const T* src = ksrc + (int64_t)(key < keys ? key : keys - 1) * a.kl;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int d = ks * 32 + 8 * quarter;
                if (WHOLE) __builtin_memcpy(r.k[x][ks], src + (d < s.D ? d : 0), 8 * sizeof(T));
                else at_words<T, 8>(src + d, s.D - d, r.k[x][ks]);
            }
        }
    };
    auto load_values = [&](int n, R& r) {
        const int key0 = tiles.at(n) * 32;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int key = key0 + key_of(e);
            const T* src = vsrc + (int64_t)(key < keys ? key : keys - 1) * a.vl;
            if (WHOLE) __builtin_memcpy(r.v[e], src + (NV * col < s.D ? NV * col : 0), NV * sizeof(T));
            else at_words<T, NV>(src + NV * col, s.D - NV * col, r.v[e]);
        }
    };
    // the next tile is on its way while one is worked on; of 16-bit elements only its keys, for which there are registers
    constexpr bool AHEAD = sizeof(T) == 1;
    R raw;
    if (begin + w < end) {
        load_keys(begin + w, raw);
        if (AHEAD) load_values(begin + w, raw);
    }

    if (K == KIND_POSIT_U8) {
        // low half: the value in bfloat16; high half: the same with zero for NaR (see AttnMarks)
        const uint32_t bits = bits_of_f32(posit_value(t, a.fkv)) >> 16;
        const uint32_t e = bits | ((bits & 0x7F80u) == 0x7F80u ? 0u : bits << 16);
#pragma unroll
        for (int c = 0; c < 8; ++c) ((uint4*)smem)[t * 8 + c] = make_uint4(e, e, e, e);
        __syncthreads();
    }
    const uint32_t* const tab = smem + (lane & 31);

    float c = s.scale * 1.4426950408889634f;
    at_v8b q[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int d = ks * 32 + 8 * quarter;
        uint4 u = make_uint4(0, 0, 0, 0);
        if (live && d < s.D) u = at_load8(a.q, b * a.qb + i * a.ql + h * a.qh + d, s.D - d, a.kq, a.fq);
        q[ks] = at_scaled(u, c);
    }
    c = at_scale(c);

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
    at_v4f o[NV];
#pragma unroll
    for (int x = 0; x < NV; ++x) o[x] = at_v4f{0.f, 0.f, 0.f, 0.f};
    uint32_t flagged = 0;
    for (int n = begin + w; n < end; n += 4) {
        if (!AHEAD) load_values(n, raw);
        const R cur = raw;
        if (n + 4 < end) {
            load_keys(n + 4, raw);
            if (AHEAD) load_values(n + 4, raw);
        }
        const int key0 = tiles.at(n) * 32;
        float sc[8];  // of keys key_of(0 .. 7)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            at_v4f acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const uint32_t* e = cur.k[x][ks];
                uint4 u = make_uint4(pair(e, 0, e, 1, false), pair(e, 2, e, 3, false), pair(e, 4, e, 5, false), pair(e, 6, e, 7, false));
                if (WHOLE && ks == KS - 1) u = ks * 32 + 8 * quarter < s.D ? u : make_uint4(0, 0, 0, 0);
                acc = at_mfma16(at_frag(u), q[ks], acc);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) sc[4 * x + r] = acc[r];
        }
        if (!(key0 + 31 <= p0 && (key0 > low1 || key0 + 31 < s.sinks))) {
#pragma unroll
            for (int r = 0; r < 8; ++r) sc[r] = at_sees(s, p, low, key0 + key_of(r)) ? sc[r] : -inf;
        }
        float mx = sc[0];
#pragma unroll
        for (int r = 1; r < 8; ++r) mx = fmaxf(mx, sc[r]);
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = at_max_halves(mx) * c;
        if (__any(mx > m + 8.f)) {
            const float m1 = fmaxf(m, mx), f = m1 == -inf ? 1.f : __builtin_amdgcn_exp2f(m - m1);
            m = m1;
            l *= f;
#pragma unroll
            for (int x = 0; x < NV; ++x) o[x] *= f;
        }
        const float mr = m == -inf ? 0.f : m;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], c, -mr));
            l += sc[r];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int x = 0; x < NV * R::B / 4; ++x) flagged |= odd(cur.v[e][x]);
        at_v8b ph, pl;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            ph[r] = (__bf16)sc[r];
            pl[r] = (__bf16)(sc[r] - (float)ph[r]);
        }
#pragma unroll
        for (int x = 0; x < NV; ++x) {
            const at_v8b v = at_frag(make_uint4(pair(cur.v[0], x, cur.v[1], x, true), pair(cur.v[2], x, cur.v[3], x, true), pair(cur.v[4], x, cur.v[5], x, true),
                                                pair(cur.v[6], x, cur.v[7], x, true)));
            o[x] = at_mfma16(v, ph, o[x]);
            o[x] = at_mfma16(v, pl, o[x]);
        }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (__any(flagged != 0)) {
        // the wave's tiles once more, an element of a value to a lane
        AttnMarks<DB> marks = {};
        for (int n = begin + w; n < end; n += 4)
#pragma unroll 4
            for (int r = 0; r < 32; ++r) {
                const int key = tiles.at(n) * 32 + r;
                const T* const src = vsrc + (int64_t)(key < keys ? key : keys - 1) * a.vl;
                uint32_t m[3][4] = {};
#pragma unroll
                for (int x = 0; x < (DB + 1) / 2; ++x) {
                    const int d = 64 * x + lane;
                    const float v = d < s.D ? value_of<K>(src[d], a.fkv) : 0.f;
                    const uint64_t b[3] = {__ballot(v == inf), __ballot(v == -inf), __ballot(v != v)};
#pragma unroll
                    for (int y = 0; y < 3; ++y) {
                        m[y][2 * x] = (uint32_t)b[y];
                        m[y][2 * x + 1] = (uint32_t)(b[y] >> 32);
                    }
                }
                marks.add(m[0], m[1], m[2], at_sees(s, p, low, key));
            }
        // the lane's elements NV (4 quarter + r) + x lie in one word
        const int word = NV * quarter / 8, from = NV * 4 * quarter & 31;
        uint32_t pos = 0, neg = 0, nan = 0;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            pos = word == d ? marks.pos[d] : pos;
            neg = word == d ? marks.neg[d] : neg;
            nan = word == d ? marks.nan[d] : nan;
        }
#pragma unroll
        for (int x = 0; x < NV; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[x][r] = at_marked(o[x][r], pos, neg, nan, from + NV * r + x);
    }

    // join the waves: a common reference, then through LDS, [wave][block][element row][column]
    if (quarter == 0) {
        wm[w][col] = m;
        wl[w][col] = l;
    }
    __syncthreads();
    const float top = fmaxf(fmaxf(wm[0][col], wm[1][col]), fmaxf(wm[2][col], wm[3][col]));
    const float f = m == -inf ? 1.f : __builtin_amdgcn_exp2f(m - top);
    float* const red = (float*)smem;
#pragma unroll
    for (int x = 0; x < NV; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float v = o[x][r];
            red[((w * NV + x) * 16 + 4 * quarter + r) * 16 + col] = v - v == 0.f ? v * f : v;  // an infinity stays one
        }
    __syncthreads();
    // NV neighbouring elements of a row to a thread
    const int rr = t >> 4, rho = t & 15, gr = rb * 16 + rr, d = NV * rho;
    if (gr >= s.rows) return;
    float out[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < NV; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) out[x] += red[((y * NV + x) * 16 + rho) * 16 + rr];
    float mm = -inf, sum = 0.f;
#pragma unroll
    for (int y = 0; y < 4; ++y) mm = fmaxf(mm, wm[y][rr]);
#pragma unroll
    for (int y = 0; y < 4; ++y) sum += wm[y][rr] == -inf ? wl[y][rr] : wl[y][rr] * __builtin_amdgcn_exp2f(wm[y][rr] - mm);
    if (a.parts > 1) {
        float* const at = a.part + ((((int64_t)b * s.HKV + hk) * (gridDim.x / a.parts) + rb) * a.parts + part) * (16 * (s.D + 2));
        if (rho == 0) {
            at[rr] = mm;
            at[16 + rr] = sum;
        }
#pragma unroll
        for (int x = 0; x < NV; ++x)
            if (d + x < s.D) at[32 + rr * s.D + d + x] = out[x];
        return;
    }
    const int gi = gr / s.G, gh = hk * s.G + (gr - gi * s.G);
    if (a.lse && rho == 0) a.lse[((int64_t)b * s.HKV * s.G + gh) * s.LQ + gi] = sum == 0.f ? -inf : mm * 0.6931471805599453f + logf(sum);
    const float up = sum == 0.f ? 0.f : 1.f / sum;
    const int64_t at = (((int64_t)b * s.LQ + gi) * (s.HKV * s.G) + gh) * s.D + d;
    const int left = s.D - d < NV ? s.D - d : NV;
#pragma unroll
    for (int x = 0; x < 8; ++x) out[x] *= up;
    at_store8(a.o, at, left, a.ko, a.fo, out);
    if (a.copy) at_store8(a.copy, at, left, a.kc, a.fc, out);
}

// Parts of a row joined, one row to a workgroup and an element to a thread; 4 to 5 us.
__global__ __launch_bounds__(128) void attn_join_kernel(AttnToken a) {
    __shared__ float weight[AT_MOST_PARTS];
    __shared__ float half_max[2], half_sum[2];
    const AttnShape& s = a.s;
    const int row = blockIdx.x, hk = blockIdx.y, b = blockIdx.z, t = threadIdx.x, rr = row & 15;
    const int i = row / s.G, h = hk * s.G + (row - i * s.G), blocks = (s.rows + 15) / 16;
    const int64_t step = 16 * (s.D + 2);
    const float* const at = a.part + (((int64_t)b * s.HKV + hk) * blocks + (row >> 4)) * a.parts * step;
    const float inf = f32_of_bits(0x7F800000u);
    float mine[AT_MOST_PARTS / 128], sums[AT_MOST_PARTS / 128], m = -inf, l = 0.f;
#pragma unroll
    for (int x = 0; x < AT_MOST_PARTS / 128; ++x) {
        const int n = t + 128 * x;
        mine[x] = n < a.parts ? at[n * step + rr] : -inf;
        sums[x] = n < a.parts ? at[n * step + 16 + rr] : 0.f;
        m = fmaxf(m, mine[x]);
    }
    m = wave_max(m);
    if ((t & 63) == 0) half_max[t >> 6] = m;
    __syncthreads();
    m = fmaxf(half_max[0], half_max[1]);
#pragma unroll
    for (int x = 0; x < AT_MOST_PARTS / 128; ++x) {
        const float f = mine[x] == -inf ? 1.f : __builtin_amdgcn_exp2f(mine[x] - m);  // a part without keys: zeros, or NaN
        weight[t + 128 * x] = f;
        l += sums[x] * f;
    }
    l = wave_sum(l);
    if ((t & 63) == 0) half_sum[t >> 6] = l;
    __syncthreads();
    l = half_sum[0] + half_sum[1];
    if (a.lse && t == 0) a.lse[((int64_t)b * s.HKV * s.G + h) * s.LQ + i] = l == 0.f ? -inf : m * 0.6931471805599453f + logf(l);
    if (t >= s.D) return;
    const float* const from = at + 32 + rr * s.D + t;
    float o = 0.f;
    for (int n = 0; n < a.parts; n += 8) {
        float v[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] = from[(n + x < a.parts ? n + x : 0) * step];
#pragma unroll
        for (int x = 0; x < 8; ++x)
            if (n + x < a.parts) o += v[x] - v[x] == 0.f ? v[x] * weight[n + x] : v[x];
    }
    const int64_t to = (((int64_t)b * s.LQ + i) * (s.HKV * s.G) + h) * s.D + t;
    o = l == 0.f ? 0.f : o / l;
    store_value(a.o, to, a.ko, a.fo, o);
    if (a.copy) store_value(a.copy, to, a.kc, a.fc, o);
}

}  // namespace pnn
