// Attention of many queries: prompts and training.
//
// A workgroup takes 128 rows (positions and heads of a group), 32 to a wave, and walks the keys that any of them sees in tiles of 64: the
// tiles of the sinks, then those of the window.  Per tile and wave, S^T = K Q^T (A: keys, B: the wave's queries, which stay in registers), so a lane
// holds 32 scores of ONE query: maximum and sum need no exchange but one between the lane's halves.  O^T += V^T P^T takes the probabilities as they
// are.  Tiles of keys and values come through LDS, two buffers, copied straight from memory while the tile before is worked on.
// What bounds it: no unit by itself (matrix 29 to 33 % of the cycles, vector 47 to 64, LDS 11 to 14), but each wave's chain from scores over maxima and
// exponentials to the second product, with 1.5 (heads of 128) to 2.8 waves on a SIMD to cover it.  2 sequences of 4001, 16 heads on 4 of 128, window 1024, to 8-bit
// posits (probabilities in two parts): 127 to 134 us, 0.69 PFLOP/s of matrix instructions; 4 of 2048, heads of 64, causal, to bfloat16: 52, 0.66;
// with a copy in binary32, so in two parts, 69.
// The running maximum is a reference: results are rescaled only when a row's maximum rises by more than 2^8 above it.
#pragma once

#include "attn_mfma.h"

namespace pnn {

struct AttnFwd {
    AttnShape s;
    const void* q;        // read once, by the wave whose rows they are
    int64_t qb, ql, qh;
    int kq;
    ElemFmt fq;
    const uint4 *k, *v;   // row fragments, transposed fragments
    void *o, *copy;
    float* lse;
    int ko, kc;
    ElemFmt fo, fc;
    int nbh;  // B * HKV
    const int32_t* flags;  // of v's blocks
    const uint4* marks;
};

// The tiles of TK keys that rows of positions p0 .. p1 see: sinks first, then the window.
struct AttnTiles {
    int head, low, count;  // tiles of sinks, first tile of the window, all
    __device__ __forceinline__ int at(int n) const { return n < head ? n : low + (n - head); }
};
template <int TK>
__device__ __forceinline__ AttnTiles at_tiles(const AttnShape& s, int p0, int p1) {
    AttnTiles t = {0, 0, 0};
    if (p1 < 0) return t;
    if (s.window && p0 - s.window + 1 > 0) {
        t.low = (p0 - s.window + 1) / TK;
        const int sinks = s.sinks < p1 + 1 ? s.sinks : p1 + 1;
        t.head = (sinks + TK - 1) / TK;
        if (t.head > t.low) t.head = t.low;
    }
    t.count = t.head + p1 / TK - t.low + 1;
    return t;
}

template <int DB, bool TWO>
__global__ __launch_bounds__(256, 2) void attn_fwd_kernel(AttnFwd a) {
    constexpr int KS = 2 * DB, RUNS = 8 * DB;  // runs of 1 KB in a tile: 4 DB of keys, 4 DB of values
    __shared__ uint4 buf[2][RUNS * 64];
    const AttnShape& s = a.s;
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), half = lane >> 5;
    // the last rows first: with a causal mask they see most
    const int bh = blockIdx.x % (unsigned)a.nbh, tile = gridDim.x / (unsigned)a.nbh - 1 - at_snake(blockIdx.x / (unsigned)a.nbh, gridDim.x / (unsigned)a.nbh, a.nbh);
    const int b = bh / s.HKV, hk = bh - b * s.HKV, base = at_keys(s, b) - s.LQ;
    const int r0 = tile * 128, rw = r0 + w * 32, row = rw + (lane & 31);
    const int last = (r0 + 128 < s.rows ? r0 + 128 : s.rows) - 1;
    const int i = row / s.G;
    const bool live = row < s.rows;
    const int p = live ? base + i : -1, low = s.window ? p - s.window : -1;
    // positions of the workgroup's and the wave's first and last row
    const AttnTiles tiles = at_tiles<64>(s, base + r0 / s.G, base + last / s.G);
    const int wlast = rw + 31 < last ? rw + 31 : last;
    const int wp0 = base + rw / s.G, wp1 = rw <= last ? base + wlast / s.G : -1;
    const int wlow0 = s.window ? wp0 - s.window : -1, wlow1 = s.window ? wp1 - s.window : -1;

    float c = s.scale * 1.4426950408889634f;
    at_v8b q[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int d = ks * 16 + 8 * half;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (live && d < s.D) v = at_load8(a.q, b * a.qb + i * a.ql + (int64_t)(hk * s.G + (row - i * s.G)) * a.qh + d, s.D - d, a.kq, a.fq);
        q[ks] = at_scaled(v, c);
    }
    c = at_scale(c);

    const uint4* const ksrc = a.k + (int64_t)bh * s.kblocks * (KS * 64);
    const uint4* const vsrc = a.v + (int64_t)bh * s.kblocks * (KS * 64);
    auto issue = [&](int n) {
        const int64_t at = (int64_t)tiles.at(n) * (2 * KS * 64);
        const uint4* src = (w < 2 ? ksrc : vsrc) + at + (w & 1) * (2 * DB * 64);
        uint4* dst = buf[n & 1] + w * (2 * DB * 64);
#pragma unroll
        for (int r = 0; r < 2 * DB; ++r) at_copy(src + r * 64, dst + r * 64, lane);
    };

    const float inf = f32_of_bits(0x7F800000u);
    float m = -inf, l = 0.f;
    at_v16f o[DB];

#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = at_zero();
    if (tiles.count > 0) issue(0);
    for (int n = 0; n < tiles.count; ++n) {
        at_landed();
        if (n + 1 < tiles.count) issue(n + 1);
        const int key0 = tiles.at(n) * 64;
        const bool any = key0 <= wp1 && (key0 + 63 > wlow0 || key0 < s.sinks);
        if (any) {
            const uint4* kb = buf[n & 1] + lane;
            const uint4* vb = kb + 4 * DB * 64;
            at_v16f sc[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                sc[x] = at_zero();
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) sc[x] = at_mfma(at_frag(kb[(x * KS + ks) * 64]), q[ks], sc[x]);
            }
            const bool whole = key0 + 63 <= wp0 && (key0 > wlow1 || key0 + 63 < s.sinks);
            if (!whole) {
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int r = 0; r < 16; ++r) sc[x][r] = at_sees(s, p, low, key0 + x * 32 + at_row(r, half)) ? sc[x][r] : -inf;
            }
            float mx = sc[0][0];
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[x][r]);
            mx = at_max_halves(mx) * c;
            if (__any(mx > m + 8.f)) {
                const float m1 = fmaxf(m, mx), f = m1 == -inf ? 1.f : __builtin_amdgcn_exp2f(m - m1);
                m = m1;
                l *= f;
#pragma unroll
                for (int d = 0; d < DB; ++d) o[d] *= f;
            }
            const float mr = m == -inf ? 0.f : m;
            float add = 0.f;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    sc[x][r] = __builtin_amdgcn_exp2f(fmaf(sc[x][r], c, -mr));
                    add += sc[x][r];
                }
            l += add;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const at_v8b ph = at_round(sc[x], 8 * y);
                    at_v8b pl;
                    if (TWO) pl = at_rest(sc[x], 8 * y, ph);
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        const at_v8b v = at_frag(vb[((2 * x + y) * DB + d) * 64]);
                        o[d] = at_mfma(v, ph, o[d]);
                        if (TWO) o[d] = at_mfma(v, pl, o[d]);
                    }
                }
        }
    }
    l += __shfl_xor(l, 32, 64);
    const int32_t* const flags = a.flags + (int64_t)bh * s.kblocks;
    bool flagged = false;
    for (int n = lane; n < tiles.count; n += 64) flagged |= (flags[2 * tiles.at(n)] | flags[2 * tiles.at(n) + 1]) != 0;
    flagged = __any(flagged);
    AttnMarks<DB> marks = {};
    if (flagged)
        marks = at_marks<DB>(
            flags, a.marks + (int64_t)bh * s.kblocks * AT_MARKS, 2 * tiles.count, false, [&](int n) { return 2 * tiles.at(n >> 1) + (n & 1); },
            [&](int blk) {
                const int key0 = blk * 32;
                if (!(key0 <= wp1 && (key0 + 31 > wlow0 || key0 < s.sinks))) return AT_NONE;
                return key0 + 31 <= wp0 && (key0 > wlow1 || key0 + 31 < s.sinks) ? AT_ALL : AT_EDGE;
            },
            [&](int key) { return at_sees(s, p, low, key); });
    if (!live) return;
    const int h = hk * s.G + (row - i * s.G);
    if (a.lse && half == 0) a.lse[((int64_t)b * s.HKV * s.G + h) * s.LQ + i] = l == 0.f ? -inf : m * 0.6931471805599453f + logf(l);
    const int64_t at = (((int64_t)b * s.LQ + i) * (s.HKV * s.G) + h) * s.D;
    const float up = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            o[d][r] *= up;
            if (flagged) o[d][r] = at_marked(o[d][r], marks.pos[d], marks.neg[d], marks.nan[d], at_row(r, half));
        }
        at_eights(o[d], half, [&](int e, const float (&v)[8]) {
            e += d * 32;
            at_store8(a.o, at + e, s.D - e, a.ko, a.fo, v);
            if (a.copy) at_store8(a.copy, at + e, s.D - e, a.kc, a.fc, v);
        });
    }
}

}  // namespace pnn
