// Gradients of attention, from recomputed probabilities: P = exp(S - lse), dS = P * (dP - D) with dP = dO V^T and D = rowsum(dO * o).
//
// Two kernels, so that every sum has one owner and a fixed order (no atomics): one walks the keys of 128 rows (dQ), as the forward kernel
// does; one walks the rows that see 64 keys (dK and dV), where the heads that share a key are rows like others.  In both
// the products that reduce over a head's elements come out in the lane order that the next product wants its operand in.
//   rows:  S^T = K Q^T and dP^T = V dO^T (a lane holds one row: lse and D are its own), dQ^T += K^T dS^T
//   keys:  S = Q K^T and dP = dO V^T (a lane holds one key), dV^T += dO^T P, dK^T += Q^T dS
// As in the forward kernel no unit is full: rows, matrix 35 % of the cycles, vector 44, LDS 17; keys 25, 27 and 20, with 1.7 waves on a SIMD (one workgroup's
// operands take most of a compute unit's LDS) that wait 39 % of their time.  4 sequences of 2048, 16 heads on 4 of 64, causal, bfloat16 out: rows 63 to 66 us, keys 116 to 122
// (0.8 and 0.6 PFLOP/s), rows' statistics 12.  TWO: P and dS go into the second products in two parts, 16 bits; for posits out, 8-bit ones for instance, rows 75 to 80, keys 146 to
// 157.  Where all gradients are bfloat16, which keeps 8 bits, they go rounded to 8: forward and backward pass 290 us rather than 331; error of the
// gradients 2.4e-3 of their size rather than 1.7e-3, which is that of their own rounding.
#pragma once

#include "attn_prompt.h"

namespace pnn {

// What the kernels need to know of each row, by blocks of 32: lse in powers of two, D, position (-1 behind the last row).
constexpr int AT_STATS = 96;

struct AttnBwd {
    AttnShape s;
    const uint4 *q, *k, *v, *g;   // row fragments
    const uint4 *qt, *kt, *gt;    // transposed fragments
    const float* stats;
    void *dq, *dk, *dv;
    int kout;
    ElemFmt fout;
    int nbh;
    const int32_t* flags;         // of d_o's blocks
    const uint4* marks;
    int parts;                    // workgroups to a tile of keys; each of them leaves its rows' sums in `part`, [part][batch, head][key][dK, dV][element]
    float* part;
};

struct AttnStats {
    AttnShape s;
    const void *g, *o;
    int64_t gb, gl, gh;
    const float* lse;
    float* stats;
    int kg, ko;
    ElemFmt fg, fo;
};

// Eight lanes to a row, 32 rows to a workgroup.
__global__ __launch_bounds__(256) void attn_stats_kernel(AttnStats a) {
    const AttnShape& s = a.s;
    const int t = threadIdx.x, blk = blockIdx.x, hk = blockIdx.y, b = blockIdx.z, r = t >> 3, row = blk * 32 + r;
    const int i = row / s.G, h = hk * s.G + (row - i * s.G), HQ = s.HKV * s.G;
    const bool live = row < s.rows;
    float d = 0.f;
    if (live) {
        const int64_t ga = b * a.gb + i * a.gl + h * a.gh, oa = (((int64_t)b * s.LQ + i) * HQ + h) * s.D;
        for (int e = (t & 7) * 8; e < s.D; e += 64) {
            Raw8 rg, ro;
            load8(rg, a.g, ga + e, a.kg, s.D - e);
            load8(ro, a.o, oa + e, a.ko, s.D - e);
            float g[8], o[8];
            values8(g, rg, a.kg, a.fg);
            values8(o, ro, a.ko, a.fo);
#pragma unroll
            for (int x = 0; x < 8; ++x) d = fmaf(g[x], o[x], d);
        }
    }
#pragma unroll
    for (int m = 4; m >= 1; m >>= 1) d += __shfl_xor(d, m, 64);
    float* const out = a.stats + (((int64_t)b * s.HKV + hk) * s.qblocks + blk) * AT_STATS + r;
    if ((t & 7) == 0) {
        out[0] = live ? a.lse[((int64_t)b * HQ + h) * s.LQ + i] * 1.4426950408889634f : 0.f;
        out[32] = d;
        out[64] = __builtin_bit_cast(float, live ? at_keys(s, b) - s.LQ + i : -1);
    }
}

template <int DB, bool TWO>
__global__ __launch_bounds__(256, 2) void attn_dq_kernel(AttnBwd a) {
    constexpr int KS = 2 * DB, RUNS = 3 * KS;  // 1 KB runs of a tile of 32 keys: keys, values, keys transposed
    __shared__ uint4 buf[2][RUNS * 64];
    const AttnShape& s = a.s;
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), half = lane >> 5;
    const int bh = blockIdx.x % (unsigned)a.nbh, tile = gridDim.x / (unsigned)a.nbh - 1 - at_snake(blockIdx.x / (unsigned)a.nbh, gridDim.x / (unsigned)a.nbh, a.nbh);
    const int b = bh / s.HKV, hk = bh - b * s.HKV, base = at_keys(s, b) - s.LQ;
    const int r0 = tile * 128, rw = r0 + w * 32, row = rw + (lane & 31);
    const int last = (r0 + 128 < s.rows ? r0 + 128 : s.rows) - 1;
    const int i = row / s.G;
    const bool live = row < s.rows;
    const int p = live ? base + i : -1, low = s.window ? p - s.window : -1;
    const AttnTiles tiles = at_tiles<32>(s, base + r0 / s.G, base + last / s.G);
    const int wlast = rw + 31 < last ? rw + 31 : last;
    const int wp0 = base + rw / s.G, wp1 = rw <= last ? base + wlast / s.G : -1;
    const int wlow0 = s.window ? wp0 - s.window : -1, wlow1 = s.window ? wp1 - s.window : -1;
    const float c = s.scale * 1.4426950408889634f;

    at_v8b q[KS], g[KS];
    const int64_t mine = (int64_t)bh * s.qblocks + tile * 4 + w;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        q[ks] = at_frag(a.q[(mine * KS + ks) * 64 + lane]);
        g[ks] = at_frag(a.g[(mine * KS + ks) * 64 + lane]);
    }
    const float lse = a.stats[mine * AT_STATS + (lane & 31)], dd = a.stats[mine * AT_STATS + 32 + (lane & 31)];

    const uint4* const src[3] = {a.k + (int64_t)bh * s.kblocks * (KS * 64), a.v + (int64_t)bh * s.kblocks * (KS * 64), a.kt + (int64_t)bh * s.kblocks * (KS * 64)};
    auto issue = [&](int n) {
        const int64_t at = (int64_t)tiles.at(n) * (KS * 64);
        uint4* dst = buf[n & 1];
#pragma unroll
        for (int x = 0; x < 3; ++x)
#pragma unroll
            for (int r = 0; r < KS; r += 4)
                if (r + w < KS) at_copy(src[x] + at + (r + w) * 64, dst + (x * KS + r + w) * 64, lane);
    };

    at_v16f dq[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dq[d] = at_zero();
    if (tiles.count > 0) issue(0);
    for (int n = 0; n < tiles.count; ++n) {
        at_landed();
        if (n + 1 < tiles.count) issue(n + 1);
        const int key0 = tiles.at(n) * 32;
        if (!(key0 <= wp1 && (key0 + 31 > wlow0 || key0 < s.sinks))) continue;
        const uint4* kb = buf[n & 1] + lane;
        at_v16f sc = at_zero(), dp = at_zero();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            sc = at_mfma(at_frag(kb[ks * 64]), q[ks], sc);
            dp = at_mfma(at_frag(kb[(KS + ks) * 64]), g[ks], dp);
        }
        const bool whole = key0 + 31 <= wp0 && (key0 > wlow1 || key0 + 31 < s.sinks);
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], c, -lse)) * (dp[r] - dd);
        if (!whole) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[r] = at_sees(s, p, low, key0 + at_row(r, half)) ? sc[r] : 0.f;
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const at_v8b sh = at_round(sc, 8 * y);
            at_v8b sl;
            if (TWO) sl = at_rest(sc, 8 * y, sh);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const at_v8b k = at_frag(kb[(2 * KS + y * DB + d) * 64]);
                dq[d] = at_mfma(k, sh, dq[d]);
                if (TWO) dq[d] = at_mfma(k, sl, dq[d]);
            }
        }
    }
    if (!live) return;
    const int64_t at = (((int64_t)b * s.LQ + i) * (s.HKV * s.G) + hk * s.G + (row - i * s.G)) * s.D;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        dq[d] *= s.scale;
        at_eights(dq[d], half, [&](int e, const float (&v)[8]) { at_store8(a.dq, at + d * 32 + e, s.D - d * 32 - e, a.kout, a.fout, v); });
    }
}

// 64 keys to a workgroup, NP blocks of 32 rows at a time: of its 2 NP waves, NP take each block of 32 keys, each with every NP-th block of
// rows, and join their sums at the end.  With a causal mask the first keys are seen by all rows and the last by few, so the length of the longest
// workgroup decides: 4 sequences of 2048, 64 elements a head, us: 128 keys and one block of rows at a time 250, 64 keys and two 164, four 115 to 122.  Both
// blocks of keys in one wave, with rows' operands straight from memory into registers, take LDS and the barriers away and come to 128: with one wave to a SIMD
// results move between the two register files.
constexpr int at_parallel(int db) { return db <= 2 ? 4 : 2; }  // what LDS (128 KB) holds of two stages

template <int DB, bool TWO>
__global__ __launch_bounds__(128 * at_parallel(DB), DB <= 2 ? 2 : 1) void attn_dkv_kernel(AttnBwd a) {
    constexpr int KS = 2 * DB, NP = at_parallel(DB), RUNS = 4 * KS;  // 1 KB runs of a block of rows: q, d_o, both transposed
    // One object for the operands and the rows' statistics behind them: between two, the compiler waits for all copies in front of the first read of
    // either, those for the next round among them.
    constexpr int ROUND = RUNS * 64 + AT_STATS / 4;
    __shared__ uint4 buf[2][NP][ROUND];
    const AttnShape& s = a.s;
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), half = lane >> 5, turn = w >> 1;
    const int bh = blockIdx.x % (unsigned)a.nbh, tile = blockIdx.x / (unsigned)a.nbh / (unsigned)a.parts, share = blockIdx.x / (unsigned)a.nbh - tile * a.parts;
    const int b = bh / s.HKV, hk = bh - b * s.HKV, keys = at_keys(s, b), base = keys - s.LQ;
    const int k0 = tile * 64, kw = k0 + (w & 1) * 32, key = kw + (lane & 31);
    const float c = s.scale * 1.4426950408889634f;
    // the rows that see any of the workgroup's keys: from the position of its first key to the end of its last key's window
    const int i0 = k0 - base > 0 ? k0 - base : 0;
    int64_t i1 = s.LQ - 1;
    if (s.window && k0 >= s.sinks && (int64_t)k0 + 62 + s.window - base < i1) i1 = (int64_t)k0 + 62 + s.window - base;
    int first = (int)((int64_t)i0 * s.G / 32), blocks = k0 >= keys || i0 > i1 ? 0 : (int)((i1 * s.G + s.G - 1) / 32) - first + 1;
    if (a.parts > 1) {  // whole rounds, the first share at the end of the rows
        const int chunk = ((blocks + a.parts - 1) / a.parts + NP - 1) / NP * NP, rest = blocks - share * chunk;
        const int mine = rest < 0 ? 0 : (rest < chunk ? rest : chunk);
        first += rest - mine;
        blocks = mine;
    }

    at_v8b kf[KS], vf[KS];
    const int64_t mine = (int64_t)bh * s.kblocks + tile * 2 + (w & 1);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        kf[ks] = at_frag(a.k[(mine * KS + ks) * 64 + lane]);
        vf[ks] = at_frag(a.v[(mine * KS + ks) * 64 + lane]);
    }
    const int64_t rows0 = (int64_t)bh * s.qblocks;
    // Blocks from the last one down: that is where the rows of all of a sequence's workgroups end, which so read the same blocks at about
    // the same time (4 MB of packed rows a sequence and head group do not fit an L2).  Each wave copies two of its own block's four operands.
    const int last = first + blocks - 1;
    const uint4* const src[2] = {((w & 1) ? a.g : a.q) + rows0 * (KS * 64), ((w & 1) ? a.gt : a.qt) + rows0 * (KS * 64)};
    auto issue = [&](int n) {
        const int blk = last - NP * n - turn;
        if (NP * n + turn >= blocks) return;
        const int64_t at = (int64_t)blk * (KS * 64);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            uint4* dst = buf[n & 1][turn] + (2 * x + (w & 1)) * (KS * 64);
#pragma unroll
            for (int r = 0; r < KS; ++r) at_copy(src[x] + at + r * 64, dst + r * 64, lane);
        }
        if ((w & 1) == 0 && lane < AT_STATS / 4) at_copy((const uint4*)(a.stats + (rows0 + blk) * AT_STATS), buf[n & 1][turn] + RUNS * 64, lane);
    };

    at_v16f dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        dk[d] = at_zero();
        dv[d] = at_zero();
    }
    if (blocks > 0) issue(0);
    const int rounds = (blocks + NP - 1) / NP;
    // row / G of the wave's block, kept up to date without a division a round
    int quot = (last - turn) * 32 / s.G, rem = (last - turn) * 32 - quot * s.G;
    const int reach = (31 + s.G - 1) / s.G;
    for (int n = 0; n < rounds; ++n) {
        at_landed();
        if (n + 1 < rounds) issue(n + 1);
        if (NP * n + turn >= blocks) continue;
        const uint4* rb = buf[n & 1][turn] + lane;
        const float* st = (const float*)(buf[n & 1][turn] + RUNS * 64) + 4 * half;
        const int row0 = (last - NP * n - turn) * 32, p0 = base + quot, p1 = p0 + reach;  // p1: the last row's position or more
        quot -= NP * 32 / s.G;
        rem -= NP * 32 % s.G;
        if (rem < 0) {
            rem += s.G;
            --quot;
        }
        const int low0 = s.window ? p0 - s.window : -1, low1 = s.window ? p1 - s.window : -1;
        if (!(kw <= p1 && (kw + 31 > low0 || kw < s.sinks))) continue;
        const bool whole = kw + 31 <= p0 && (kw > low1 || kw + 31 < s.sinks) && row0 + 31 < s.rows;
        at_v16f sc = at_zero(), dp = at_zero();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            sc = at_mfma(at_frag(rb[ks * 64]), kf[ks], sc);
            dp = at_mfma(at_frag(rb[(KS + ks) * 64]), vf[ks], dp);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], c, -st[at_row(r, 0)]));
            dp[r] -= st[32 + at_row(r, 0)];
        }
        if (!whole) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int p = __builtin_bit_cast(int, st[64 + at_row(r, 0)]);
                const bool see = at_sees(s, p, s.window ? p - s.window : -1, key);
                sc[r] = see ? sc[r] : 0.f;
                dp[r] = see ? dp[r] : 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] *= sc[r];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const at_v8b ph = at_round(sc, 8 * y), sh = at_round(dp, 8 * y);
            at_v8b pl, sl;
            if (TWO) {
                pl = at_rest(sc, 8 * y, ph);
                sl = at_rest(dp, 8 * y, sh);
            }
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const at_v8b qt = at_frag(rb[(2 * KS + y * DB + d) * 64]), gt = at_frag(rb[(3 * KS + y * DB + d) * 64]);
                dv[d] = at_mfma(gt, ph, dv[d]);
                dk[d] = at_mfma(qt, sh, dk[d]);
                if (TWO) {
                    dv[d] = at_mfma(gt, pl, dv[d]);
                    dk[d] = at_mfma(qt, sl, dk[d]);
                }
            }
        }
    }
    // turn 0 finishes dK, turn 1 dV
    __syncthreads();
    {
        constexpr int PART = DB * 1024;  // floats of one wave's dK or dV
        float* const mine = (float*)buf + (w & 1) * (NP * 2 * PART) + lane;
        auto slot = [&](int of, int what, int d, int r) -> float& { return mine[(of * 2 + what) * PART + (d * 16 + r) * 64]; };
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if (turn != 0) slot(turn, 0, d, r) = dk[d][r];
                if (turn != 1) slot(turn, 1, d, r) = dv[d][r];
            }
        __syncthreads();
        if (turn > 1) return;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float v = turn == 0 ? dk[d][r] : slot(0, 1, d, r);
                v += turn == 0 ? slot(1, 0, d, r) : dv[d][r];
#pragma unroll
                for (int x = 2; x < NP; ++x) v += slot(x, turn, d, r);
                dk[d][r] = v;
            }
    }
    bool flagged = false;
    for (int n = lane; n < blocks && turn == 1; n += 64) flagged |= a.flags[rows0 + first + n] != 0;
    flagged = __any(flagged);
    AttnMarks<DB> marks = {};
    if (flagged)
        marks = at_marks<DB>(
            a.flags + rows0, a.marks + rows0 * AT_MARKS, blocks, key < s.sinks, [&](int n) { return first + n; },
            [&](int blk) {
                const int p0 = base + blk * 32 / s.G, p1 = base + (blk * 32 + 31) / s.G;  // p1: the last row's position or more
                const int low0 = s.window ? p0 - s.window : -1, low1 = s.window ? p1 - s.window : -1;
                if (!(kw <= p1 && (kw + 31 > low0 || kw < s.sinks))) return AT_NONE;
                if (kw + 31 > p0) return AT_EDGE;
                return kw > low1 || kw + 31 < s.sinks ? AT_ALL : (kw + 31 <= low0 ? AT_SINKS : AT_EDGE);
            },
            [&](int row) {
                const int p = base + row / s.G;
                return row < s.rows && at_sees(s, p, s.window ? p - s.window : -1, key);
            });
    if (key >= s.LK) return;
    const int64_t at = a.parts > 1 ? (((share * (int64_t)a.nbh + bh) * s.LK + key) * 2 + turn) * s.D : (((int64_t)b * s.LK + key) * s.HKV + hk) * s.D;
    void* const out = a.parts > 1 ? a.part : (turn ? a.dv : a.dk);
    const int kind = a.parts > 1 ? KIND_F32 : a.kout;
    const float up = turn ? 1.f : s.scale;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            dk[d][r] *= up;
            if (flagged) dk[d][r] = at_marked(dk[d][r], marks.pos[d], marks.neg[d], marks.nan[d], at_row(r, half));
        }
        at_eights(dk[d], half, [&](int e, const float (&v)[8]) { at_store8(out, at + d * 32 + e, s.D - d * 32 - e, kind, a.fout, v); });
    }
}

// The shares of a tile's rows added up, an element of dK or dV to a thread.
__global__ __launch_bounds__(256) void attn_dkv_join_kernel(AttnBwd a) {
    const AttnShape& s = a.s;
    const int64_t n = (int64_t)a.nbh * s.LK * 2 * s.D, x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (x >= n) return;
    float v = 0.f;
    for (int y = 0; y < a.parts; ++y) v += a.part[y * n + x];
    const int64_t row = x / s.D, key = (row >> 1) % s.LK, bh = (row >> 1) / s.LK, b = bh / s.HKV, hk = bh - b * s.HKV;
    store_value((row & 1) ? a.dv : a.dk, ((b * s.LK + key) * s.HKV + hk) * s.D + (x - row * s.D), a.kout, a.fout, v);
}

}  // namespace pnn
