// posit_attention_fwd / posit_attention_bwd: attention with a sliding window and sinks.
#include "attn_bwd.h"
#include "attn_token.h"

namespace pnn {

// formats that bfloat16 holds exactly: at most 8 significant bits
inline int operand_status(int f) {
    if (const int s = element_status(f)) return s;
    return f == PNN_POSIT16_1 || f == PNN_POSIT12_1 || f == PNN_F32 ? PNN_EUNSUPPORTED : PNN_OK;
}

inline int desc_status(const pnn_attention_desc* d) {
    if (!d || d->B < 0 || d->HQ < 0 || d->HKV < 0 || d->LQ < 0 || d->LK < 0 || d->D < 0 || d->window < 0 || d->sinks < 0) return PNN_EINVAL;
    if ((d->HKV == 0) != (d->HQ == 0) || (d->HKV > 0 && d->HQ % d->HKV != 0)) return PNN_EINVAL;
    if (!(d->scale > -3.4028235e38f && d->scale < 3.4028235e38f)) return PNN_EINVAL;
    if (d->qb < 0 || d->ql < 0 || d->qh < 0 || d->kb < 0 || d->kl < 0 || d->kh < 0 || d->vb < 0 || d->vl < 0 || d->vh < 0) return PNN_EINVAL;
    // rows of a group and keys are counted in 32 bits, workgroups by the grid's limits (along x: see launches())
    const int64_t most = ((int64_t)1 << 31) - 128;
    if (d->D > 128 || d->LQ > most || d->LK > most || d->HQ >= 65536 || d->B >= 16384) return PNN_EUNSUPPORTED;
    if (d->HKV > 0 && d->LQ * (d->HQ / d->HKV) > most) return PNN_EUNSUPPORTED;
    if (d->HKV > 0 && d->B * d->HKV * ((d->LQ * (d->HQ / d->HKV) + 127) / 128 + 1) > most) return PNN_EUNSUPPORTED;
    return PNN_OK;
}

}  // namespace pnn

using namespace pnn;

namespace {

int64_t up128(int64_t n) { return (n + 127) / 128 * 128; }

// Sizes that both passes use: heads of a group side by side, a head's elements padded to blocks of 32, rows and keys to 128.
struct Plan {
    AttnShape s;
    int db;
    int64_t nbh, q_bytes, k_bytes;  // of one packed operand
};

// Few queries on many keys go to the token kernel: it decodes a cache where it reads it and splits its length over workgroups; the
// prompt kernel reads a packed copy and has a workgroup to 128 rows.  The token kernel reads and decodes the cache once for each 16 rows.  us, token and prompt kernel, heads of
// 128: 16 rows a group, 8 groups of 8-bit posits, 128 keys 9 and 16, 4096 keys 17 and 102; 384 groups, 12 and 33, 117 and 530.  64 rows, 8 groups, 512 keys 16 and 25, 4096 25
// and 107; 384 groups 53 and 72, 303 and 540; bfloat16, 384 groups, 65 and 60, 460 and 462: there the two meet.  Beyond 64 rows the better one depends on the number of groups, too: 96
// rows of bfloat16, 4096 keys, 384 groups 665 and 466, but 8 groups 34 and 101.
struct TokenPlan {
    bool use;
    int blocks, parts, tiles;  // row blocks of 16, parts of the keys, tiles of 32 keys in a part
    int64_t bytes;
};

// From make_plan's sizes: window and sinks there are at most the keys, so that their sum is small.
TokenPlan token_plan(const AttnShape& s, int64_t B) {
    TokenPlan t = {};
    const int64_t rows = s.rows;
    t.use = rows <= 16 || (rows <= 64 && s.LK >= 8 * rows);
    if (!t.use) return t;
    t.blocks = (int)((rows + 15) / 16);
    int64_t keys = s.LK;
    if (s.window > 0 && (int64_t)s.window + s.LQ + s.sinks + 64 < keys) keys = (int64_t)s.window + s.LQ + s.sinks + 64;
    const int64_t all = (keys + 31) / 32 + 1, groups = B * s.HKV * t.blocks;
    // Two workgroups to a compute unit, at least a tile to each of their waves; short caches stay whole, the second kernel costs more.  48 sequences of
    // 4096 keys, 8 heads of 128: 112 us in 2 parts, 110 in 3, 124 in 4; 8 sequences of 8192: 47 in 8 parts, 52 in 16, 59 in 24.
    int64_t parts = groups > 0 ? (512 + groups - 1) / groups : 1;
    if (parts > all / 4) parts = all / 4;
    if (parts > AT_MOST_PARTS) parts = AT_MOST_PARTS;
    if (parts < 1 || all <= 16) parts = 1;
    t.tiles = (int)((all + parts - 1) / parts);
    t.tiles = (t.tiles + 3) / 4 * 4;
    t.parts = (int)((all + t.tiles - 1) / t.tiles);
    t.bytes = t.parts > 1 ? groups * t.parts * 16 * (s.D + 2) * 4 : 0;
    return t;
}

Plan make_plan(const pnn_attention_desc& d) {
    Plan p;
    p.s.LQ = (int)d.LQ; p.s.LK = (int)d.LK; p.s.lens = nullptr;
    p.s.window = d.window >= d.LK ? 0 : (int)d.window;  // a window of all keys is none
    p.s.sinks = (int)(d.sinks < d.LK ? d.sinks : d.LK);
    p.s.HKV = (int)d.HKV; p.s.G = d.HKV ? (int)(d.HQ / d.HKV) : 1; p.s.D = (int)d.D; p.s.scale = d.scale;
    p.s.rows = (int)(d.LQ * p.s.G);
    p.s.qblocks = (int)(up128(p.s.rows) / 32);
    p.s.kblocks = (int)(up128(d.LK) / 32);
    p.db = (int)((d.D + 31) / 32);
    p.nbh = d.B * d.HKV;
    p.q_bytes = p.nbh * p.s.qblocks * 2048 * p.db;
    p.k_bytes = p.nbh * p.s.kblocks * 2048 * p.db;
    return p;
}

// Workgroups to a tile of 64 keys in the backward pass: one holds a compute unit's LDS, so where tiles are fewer than half the chip's units their rows are
// shared out, at least two rounds of blocks to a workgroup (forward and backward pass of 2 sequences of 976, 4 heads on one of 40, window 53: 95 us, now 58;
// of 840, 4 on one of 64, causal: 97 and 76).
int dkv_parts(const Plan& p) {
    const int64_t tiles = p.nbh * (p.s.kblocks / 2), rounds = p.s.qblocks / at_parallel(p.db);
    if (tiles == 0) return 1;
    int64_t parts = 256 / tiles;
    if (parts > rounds / 2) parts = rounds / 2;
    return parts > 1 ? (int)parts : 1;
}
int64_t dkv_part_bytes(const Plan& p) {
    const int parts = dkv_parts(p);
    return parts > 1 ? parts * p.nbh * p.s.LK * 2 * p.s.D * 4 : 0;
}

// whether every launch's threads can be counted
bool launches(int which, const Plan& p) {
    const int64_t most = most_workgroups(256);
    if (p.nbh * (p.s.qblocks / 4) > most || p.s.kblocks > most) return false;
    return which == 0 || (p.s.qblocks <= most && p.nbh * (p.s.kblocks / 2) * dkv_parts(p) <= most_workgroups(128 * at_parallel(p.db)));
}

void launch_pack(hipStream_t st, const Plan& p, const AttnPack& a, int items) {
    int64_t blocks = 0;
    for (int i = 0; i < items; ++i) blocks = a.item[i].blocks > blocks ? a.item[i].blocks : blocks;
    if (blocks == 0) return;
    const dim3 grid((unsigned)blocks, (unsigned)a.HKV, (unsigned)(items * a.B));
    switch (p.db) {
        case 1: hipLaunchKernelGGL(attn_pack_kernel<1>, grid, dim3(256), 0, st, a); break;
        case 2: hipLaunchKernelGGL(attn_pack_kernel<2>, grid, dim3(256), 0, st, a); break;
        case 3: hipLaunchKernelGGL(attn_pack_kernel<3>, grid, dim3(256), 0, st, a); break;
        default: hipLaunchKernelGGL(attn_pack_kernel<4>, grid, dim3(256), 0, st, a); break;
    }
}

template <bool TWO>
void launch_fwd(hipStream_t st, const Plan& p, const AttnFwd& a) {
    const dim3 grid((unsigned)(p.nbh * (p.s.qblocks / 4)));
    switch (p.db) {
        case 1: hipLaunchKernelGGL((attn_fwd_kernel<1, TWO>), grid, dim3(256), 0, st, a); break;
        case 2: hipLaunchKernelGGL((attn_fwd_kernel<2, TWO>), grid, dim3(256), 0, st, a); break;
        case 3: hipLaunchKernelGGL((attn_fwd_kernel<3, TWO>), grid, dim3(256), 0, st, a); break;
        default: hipLaunchKernelGGL((attn_fwd_kernel<4, TWO>), grid, dim3(256), 0, st, a); break;
    }
}

template <int DB, bool TWO>
void launch_bwd_of(hipStream_t st, const Plan& p, const AttnBwd& a) {
    if (p.s.LQ > 0) hipLaunchKernelGGL((attn_dq_kernel<DB, TWO>), dim3((unsigned)(p.nbh * (p.s.qblocks / 4))), dim3(256), 0, st, a);
    if (p.s.LK == 0) return;
    hipLaunchKernelGGL((attn_dkv_kernel<DB, TWO>), dim3((unsigned)(p.nbh * (p.s.kblocks / 2) * a.parts)), dim3(128 * at_parallel(DB)), 0, st, a);
    if (a.parts > 1) hipLaunchKernelGGL(attn_dkv_join_kernel, dim3((unsigned)((p.nbh * p.s.LK * 2 * p.s.D + 255) / 256)), dim3(256), 0, st, a);
}

template <bool TWO>
void launch_bwd(hipStream_t st, const Plan& p, const AttnBwd& a) {
    switch (p.db) {
        case 1: launch_bwd_of<1, TWO>(st, p, a); break;
        case 2: launch_bwd_of<2, TWO>(st, p, a); break;
        case 3: launch_bwd_of<3, TWO>(st, p, a); break;
        default: launch_bwd_of<4, TWO>(st, p, a); break;
    }
}

template <int K>
void launch_token(hipStream_t st, int db, const dim3& grid, const AttnToken& a) {
    const bool whole = a.s.D % 8 == 0;
#define PNN_TOKEN(DB)                                                                                   \
    if (whole) hipLaunchKernelGGL((attn_token_kernel<K, DB, true>), grid, dim3(256), 0, st, a);         \
    else hipLaunchKernelGGL((attn_token_kernel<K, DB, false>), grid, dim3(256), 0, st, a);
    switch (db) {
        case 1: PNN_TOKEN(1) break;
        case 2: PNN_TOKEN(2) break;
        case 3: PNN_TOKEN(3) break;
        default: PNN_TOKEN(4) break;
    }
#undef PNN_TOKEN
}

}  // namespace

extern "C" size_t posit_attention_workspace(int which, int fkv, const pnn_attention_desc* desc) {
    if (desc_status(desc) || desc->B == 0 || desc->HQ == 0 || desc->D == 0) return 0;
    const Plan p = make_plan(*desc);
    const TokenPlan t = token_plan(p.s, desc->B);
    if (which == 0 && t.use) return (size_t)t.bytes;
    if (!launches(which, p)) return 0;
    if (which == 0) return (size_t)(2 * p.k_bytes + p.nbh * p.s.kblocks * (AT_MARKS * 16 + 4));
    return (size_t)(4 * p.q_bytes + 3 * p.k_bytes + p.nbh * p.s.qblocks * (AT_STATS * 4 + AT_MARKS * 16 + 4) + dkv_part_bytes(p));
}

extern "C" int posit_attention_fwd(void* stream, int fq, int fkv, int fout, const pnn_attention_desc* desc, const void* q, const void* k, const void* v,
                                   const int32_t* lens, void* o, float* lse, int fcopy, void* o_copy, void* workspace, size_t workspace_bytes) {
    if (const int s = desc_status(desc)) return s;
    for (int f : {fq, fkv})
        if (const int s = operand_status(f)) return s;
    for (int f : {fout, o_copy ? fcopy : fout})
        if (const int s = element_status(f)) return s;
    const pnn_attention_desc& d = *desc;
    if (d.B == 0 || d.HQ == 0 || d.LQ == 0 || d.D == 0) return PNN_OK;
    if (!q || !o || (d.LK > 0 && (!k || !v))) return PNN_EINVAL;
    Plan p = make_plan(d);
    p.s.lens = lens;
    const TokenPlan tp = token_plan(p.s, d.B);
    if (!tp.use && !launches(0, p)) return PNN_EUNSUPPORTED;
    const size_t need = posit_attention_workspace(0, fkv, desc);
    if (need > 0 && (!workspace || workspace_bytes < need)) return PNN_EWORKSPACE;
    if (need > 0 && !aligned(workspace, 16)) return PNN_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    discard_stale_hip_error();
    if (tp.use) {
        AttnToken a = {};
        a.s = p.s; a.q = q; a.k = k; a.v = v;
        a.qb = d.qb; a.ql = d.ql; a.qh = d.qh; a.kb = d.kb; a.kl = d.kl; a.kh = d.kh; a.vb = d.vb; a.vl = d.vl; a.vh = d.vh;
        a.kq = kind_of(fq); a.fq = elem_fmt(fq); a.fkv = elem_fmt(fkv);
        a.o = o; a.copy = o_copy; a.lse = lse; a.ko = kind_of(fout); a.fo = elem_fmt(fout); a.kc = kind_of(o_copy ? fcopy : fout); a.fc = elem_fmt(o_copy ? fcopy : fout);
        a.tiles = tp.tiles; a.parts = tp.parts; a.part = (float*)workspace;
        const dim3 grid((unsigned)(tp.blocks * tp.parts), (unsigned)d.HKV, (unsigned)d.B);
        switch (kind_of(fkv)) {
            case KIND_POSIT_U8: launch_token<KIND_POSIT_U8>(st, p.db, grid, a); break;
            case KIND_POSIT_U16: launch_token<KIND_POSIT_U16>(st, p.db, grid, a); break;
            default: launch_token<KIND_BF16>(st, p.db, grid, a); break;
        }
        if (tp.parts > 1) hipLaunchKernelGGL(attn_join_kernel, dim3((unsigned)p.s.rows, (unsigned)d.HKV, (unsigned)d.B), dim3(128), 0, st, a);
        return hip_status(hipGetLastError());
    }
    uint4* const wk = (uint4*)workspace;
    uint4* const wv = wk + p.k_bytes / 16;
    uint4* const marks = wv + p.k_bytes / 16;
    int32_t* const flags = (int32_t*)(marks + p.nbh * p.s.kblocks * AT_MARKS);
    AttnPack pack = {};
    pack.B = (int)d.B; pack.HKV = (int)d.HKV; pack.D = (int)d.D;
    pack.item[0] = {k, d.kb, d.kl, d.kh, p.s.LK, p.s.kblocks, wk, nullptr, 1, kind_of(fkv), elem_fmt(fkv), nullptr, nullptr};
    pack.item[1] = {v, d.vb, d.vl, d.vh, p.s.LK, p.s.kblocks, nullptr, wv, 1, kind_of(fkv), elem_fmt(fkv), flags, marks};
    launch_pack(st, p, pack, 2);
    AttnFwd a = {};
    a.s = p.s; a.q = q; a.qb = d.qb; a.ql = d.ql; a.qh = d.qh; a.kq = kind_of(fq); a.fq = elem_fmt(fq); a.k = wk; a.v = wv; a.o = o; a.copy = o_copy; a.lse = lse;
    a.ko = kind_of(fout); a.fo = elem_fmt(fout); a.kc = kind_of(o_copy ? fcopy : fout); a.fc = elem_fmt(o_copy ? fcopy : fout);
    a.nbh = (int)p.nbh;
    a.flags = flags; a.marks = marks;
    // The probabilities to 16 bits where an output's format keeps more than 8.  In the copy that the backward pass reads, what the rounding to 8 takes from
    // a row is common to all its gradients of scores (error of dq 2.6e-3 rather than 2.4e-3, 1.7e-3 of it its own rounding to bfloat16).  With bfloat16 outputs alone, 8
    // bits: 4 sequences of 2048, 16 heads on 4 of 64, 64 us rather than 82, error of o 2.1e-3 rather than 1.6e-3.
    if (fout != PNN_BF16 || (o_copy && fcopy != PNN_BF16)) launch_fwd<true>(st, p, a);
    else launch_fwd<false>(st, p, a);
    return hip_status(hipGetLastError());
}

extern "C" int posit_attention_bwd(void* stream, int fd, int fq, int fkv, int fo, int fout, const pnn_attention_desc* desc, const void* d_o, const void* q,
                                   const void* k, const void* v, const int32_t* lens, const void* o, const float* lse, void* dq, void* dk, void* dv,
                                   void* workspace, size_t workspace_bytes) {
    if (const int s = desc_status(desc)) return s;
    for (int f : {fd, fq, fkv})
        if (const int s = operand_status(f)) return s;
    for (int f : {fo, fout})
        if (const int s = element_status(f)) return s;
    const pnn_attention_desc& d = *desc;
    if (d.B == 0 || d.HQ == 0 || d.D == 0 || (d.LQ == 0 && d.LK == 0)) return PNN_OK;
    if ((d.LQ > 0 && (!d_o || !q || !o || !lse || !dq)) || (d.LK > 0 && (!k || !v || !dk || !dv))) return PNN_EINVAL;
    Plan p = make_plan(d);
    p.s.lens = lens;
    if (!launches(1, p)) return PNN_EUNSUPPORTED;
    const size_t need = posit_attention_workspace(1, fkv, desc);
    if (need > 0 && (!workspace || workspace_bytes < need)) return PNN_EWORKSPACE;
    if (need > 0 && !aligned(workspace, 16)) return PNN_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    discard_stale_hip_error();
    const int64_t nq = p.q_bytes / 16, nk = p.k_bytes / 16;
    uint4* const at = (uint4*)workspace;
    uint4 *wq = at, *wg = at + nq, *wqt = at + 2 * nq, *wgt = at + 3 * nq, *wk = at + 4 * nq, *wv = wk + nk, *wkt = wk + 2 * nk;
    float* const stats = (float*)(wk + 3 * nk);
    uint4* const marks = (uint4*)(stats + p.nbh * p.s.qblocks * AT_STATS);
    int32_t* const flags = (int32_t*)(marks + p.nbh * p.s.qblocks * AT_MARKS);
    AttnPack pack = {};
    pack.B = (int)d.B; pack.HKV = (int)d.HKV; pack.D = (int)d.D;
    pack.item[0] = {q, d.qb, d.ql, d.qh, p.s.rows, p.s.qblocks, wq, wqt, p.s.G, kind_of(fq), elem_fmt(fq), nullptr, nullptr};
    pack.item[1] = {d_o, d.qb, d.ql, d.qh, p.s.rows, p.s.qblocks, wg, wgt, p.s.G, kind_of(fd), elem_fmt(fd), flags, marks};
    pack.item[2] = {k, d.kb, d.kl, d.kh, p.s.LK, p.s.kblocks, wk, wkt, 1, kind_of(fkv), elem_fmt(fkv), nullptr, nullptr};
    pack.item[3] = {v, d.vb, d.vl, d.vh, p.s.LK, p.s.kblocks, wv, nullptr, 1, kind_of(fkv), elem_fmt(fkv), nullptr, nullptr};
    launch_pack(st, p, pack, 4);
    if (d.LQ > 0) {
        AttnStats c = {};
        c.s = p.s; c.g = d_o; c.o = o; c.gb = d.qb; c.gl = d.ql; c.gh = d.qh; c.lse = lse; c.stats = stats;
        c.kg = kind_of(fd); c.fg = elem_fmt(fd); c.ko = kind_of(fo); c.fo = elem_fmt(fo);
        hipLaunchKernelGGL(attn_stats_kernel, dim3((unsigned)p.s.qblocks, (unsigned)d.HKV, (unsigned)d.B), dim3(256), 0, st, c);
    }
    AttnBwd a = {};
    a.s = p.s; a.q = wq; a.g = wg; a.qt = wqt; a.gt = wgt; a.k = wk; a.v = wv; a.kt = wkt; a.stats = stats; a.dq = dq; a.dk = dk; a.dv = dv;
    a.kout = kind_of(fout); a.fout = elem_fmt(fout); a.nbh = (int)p.nbh;
    a.parts = dkv_parts(p); a.part = (float*)(flags + p.nbh * p.s.qblocks);
    a.flags = flags; a.marks = marks;
    // probabilities and score gradients to 8 bits for bfloat16 gradients, else to 16 (both sides: attn_bwd.h)
    if (fout == PNN_BF16) launch_bwd<false>(st, p, a);
    else launch_bwd<true>(st, p, a);
    return hip_status(hipGetLastError());
}
