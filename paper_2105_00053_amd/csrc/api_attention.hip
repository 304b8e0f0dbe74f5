// posit_attention_fwd / posit_attention_bwd: attention with a sliding window and sinks.
#include "attn_prompt.h"

namespace pnn {

struct Attn {
    pnn_attention_desc d;
    const void *q, *k, *v, *o, *d_o;
    const int32_t* lens;
    void *out, *copy, *dq, *dk, *dv;
    float* lse;
    const float* lse_in;
    int kq, kkv, kout, kcopy, kd, ko;
    ElemFmt fq, fkv, fout, fcopy, fd, fo;
};

__device__ __forceinline__ int64_t keys_of(const Attn& a, int64_t b) {
    const int64_t n = a.lens ? a.lens[b] : a.d.LK;
    return n < 0 ? 0 : (n > a.d.LK ? a.d.LK : n);
}
__device__ __forceinline__ bool sees(const Attn& a, int64_t p, int64_t j) { return j <= p && (a.d.window == 0 || j > p - a.d.window || j < a.d.sinks); }

__device__ __forceinline__ float row_dot(const Attn& a, int64_t qat, const void* x, int kx, ElemFmt fx, int64_t kat, const void* y) {
    float s = 0.f;
    for (int c = 0; c < a.d.D; ++c) s = fmaf(load_value(x, qat + c, kx, fx), load_value(y, kat + c, a.kkv, a.fkv), s);
    return s;
}

__device__ __forceinline__ float dot_with_o(const Attn& a, int64_t b, int64_t i, int64_t h) {
    const pnn_attention_desc& d = a.d;
    float s = 0.f;
    for (int c = 0; c < d.D; ++c)
        s = fmaf(load_value(a.d_o, b * d.qb + i * d.ql + h * d.qh + c, a.kd, a.fd), load_value(a.o, ((b * d.LQ + i) * d.HQ + h) * d.D + c, a.ko, a.fo), s);
    return s;
}

__global__ __launch_bounds__(64) void attn_dq_simple(Attn a) {
    __shared__ float ds[64];
    const pnn_attention_desc& d = a.d;
    const int64_t i = blockIdx.x, h = blockIdx.y, b = blockIdx.z, hk = h / (d.HQ / d.HKV);
    const int t = threadIdx.x;
    const int64_t p = keys_of(a, b) - d.LQ + i, qat = b * d.qb + i * d.ql + h * d.qh;
    const float lse = a.lse_in[(b * d.HQ + h) * d.LQ + i], dd = dot_with_o(a, b, i, h);
    float g[2] = {0.f, 0.f};
    for (int64_t j0 = 0; j0 <= p; j0 += 64) {
        const int64_t j = j0 + t;
        float e = 0.f;
        if (j <= p && sees(a, p, j)) {
            const float s = row_dot(a, qat, a.q, a.kq, a.fq, b * d.kb + j * d.kl + hk * d.kh, a.k) * d.scale;
            e = expf(s - lse) * (row_dot(a, qat, a.d_o, a.kd, a.fd, b * d.vb + j * d.vl + hk * d.vh, a.v) - dd) * d.scale;
        }
        __syncthreads();
        ds[t] = e;
        __syncthreads();
        for (int c = 0; c < 2; ++c)
            if (t + 64 * c < d.D)
                for (int jj = 0; jj < 64 && j0 + jj <= p; ++jj)
                    if (sees(a, p, j0 + jj)) g[c] = fmaf(ds[jj], load_value(a.k, b * d.kb + (j0 + jj) * d.kl + hk * d.kh + t + 64 * c, a.kkv, a.fkv), g[c]);
    }
    for (int c = 0; c < 2; ++c)
        if (t + 64 * c < d.D) store_value(a.dq, ((b * d.LQ + i) * d.HQ + h) * d.D + t + 64 * c, a.kout, a.fout, g[c]);
}

// One wave to a key: 64 queries at a time, over the heads that share it.
__global__ __launch_bounds__(64) void attn_dkv_simple(Attn a) {
    __shared__ float ps[64], ds[64];
    const pnn_attention_desc& d = a.d;
    const int64_t j = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
    const int t = threadIdx.x;
    const int64_t n = keys_of(a, b), G = d.HQ / d.HKV;
    float gk[2] = {0.f, 0.f}, gv[2] = {0.f, 0.f};
    for (int64_t h = hk * G; h < hk * G + G; ++h)
        for (int64_t i0 = 0; i0 < d.LQ && j < n; i0 += 64) {
            const int64_t i = i0 + t, p = n - d.LQ + i, qat = b * d.qb + i * d.ql + h * d.qh;
            float e = 0.f, w = 0.f;
            if (i < d.LQ && sees(a, p, j)) {
                const float s = row_dot(a, qat, a.q, a.kq, a.fq, b * d.kb + j * d.kl + hk * d.kh, a.k) * d.scale;
                w = expf(s - a.lse_in[(b * d.HQ + h) * d.LQ + i]);
                e = w * (row_dot(a, qat, a.d_o, a.kd, a.fd, b * d.vb + j * d.vl + hk * d.vh, a.v) - dot_with_o(a, b, i, h)) * d.scale;
            }
            __syncthreads();
            ps[t] = w;
            ds[t] = e;
            __syncthreads();
            for (int c = 0; c < 2; ++c)
                if (t + 64 * c < d.D)
                    for (int ii = 0; ii < 64 && i0 + ii < d.LQ; ++ii)
                        if (sees(a, n - d.LQ + i0 + ii, j)) {
                            const int64_t at = b * d.qb + (i0 + ii) * d.ql + h * d.qh + t + 64 * c;
                            gk[c] = fmaf(ds[ii], load_value(a.q, at, a.kq, a.fq), gk[c]);
                            gv[c] = fmaf(ps[ii], load_value(a.d_o, at, a.kd, a.fd), gv[c]);
                        }
        }
    for (int c = 0; c < 2; ++c)
        if (t + 64 * c < d.D) {
            const int64_t at = ((b * d.LK + j) * d.HKV + hk) * d.D + t + 64 * c;
            store_value(a.dk, at, a.kout, a.fout, gk[c]);
            store_value(a.dv, at, a.kout, a.fout, gv[c]);
        }
}

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
    // rows of a group and keys are counted in 32 bits, workgroups by the grid's limits
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

}  // namespace

extern "C" size_t posit_attention_workspace(int which, int fkv, const pnn_attention_desc* desc) {
    if (desc_status(desc) || desc->B == 0 || desc->HQ == 0 || desc->D == 0) return 0;
    const Plan p = make_plan(*desc);
    return which == 0 ? (size_t)(p.q_bytes + 2 * p.k_bytes + p.nbh * p.s.kblocks * 4) : 0;
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
    const size_t need = posit_attention_workspace(0, fkv, desc);
    if (need > 0 && (!workspace || workspace_bytes < need)) return PNN_EWORKSPACE;
    if (need > 0 && !aligned(workspace, 16)) return PNN_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    discard_stale_hip_error();
    Plan p = make_plan(d);
    p.s.lens = lens;
    uint4* const wq = (uint4*)workspace;
    uint4* const wk = wq + p.q_bytes / 16;
    uint4* const wv = wk + p.k_bytes / 16;
    int32_t* const flags = (int32_t*)(wv + p.k_bytes / 16);
    AttnPack pack = {};
    pack.B = (int)d.B; pack.HKV = (int)d.HKV; pack.D = (int)d.D;
    pack.item[0] = {q, d.qb, d.ql, d.qh, p.s.rows, p.s.qblocks, wq, nullptr, p.s.G, kind_of(fq), elem_fmt(fq), nullptr};
    pack.item[1] = {k, d.kb, d.kl, d.kh, p.s.LK, p.s.kblocks, wk, nullptr, 1, kind_of(fkv), elem_fmt(fkv), nullptr};
    pack.item[2] = {v, d.vb, d.vl, d.vh, p.s.LK, p.s.kblocks, nullptr, wv, 1, kind_of(fkv), elem_fmt(fkv), flags};
    launch_pack(st, p, pack, 3);
    AttnFwd a = {};
    a.s = p.s; a.q = wq; a.k = wk; a.v = wv; a.o = o; a.copy = o_copy; a.lse = lse;
    a.ko = kind_of(fout); a.fo = elem_fmt(fout); a.kc = kind_of(o_copy ? fcopy : fout); a.fc = elem_fmt(o_copy ? fcopy : fout);
    a.nbh = (int)p.nbh;
    a.flags = flags; a.vsrc = v; a.vb = d.vb; a.vl = d.vl; a.vh = d.vh; a.kv = kind_of(fkv); a.fv = elem_fmt(fkv);
    if (fout == PNN_BF16 && (!o_copy || fcopy == PNN_BF16)) launch_fwd<false>(st, p, a);
    else launch_fwd<true>(st, p, a);
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
    discard_stale_hip_error();
    Attn a = {};
    a.d = d; a.q = q; a.k = k; a.v = v; a.d_o = d_o; a.o = o; a.lse_in = lse; a.lens = lens; a.dq = dq; a.dk = dk; a.dv = dv;
    a.kq = kind_of(fq); a.fq = elem_fmt(fq); a.kkv = kind_of(fkv); a.fkv = elem_fmt(fkv); a.kout = kind_of(fout); a.fout = elem_fmt(fout);
    a.kd = kind_of(fd); a.fd = elem_fmt(fd); a.ko = kind_of(fo); a.fo = elem_fmt(fo);
    if (d.LQ > 0) hipLaunchKernelGGL(attn_dq_simple, dim3((unsigned)d.LQ, (unsigned)d.HQ, (unsigned)d.B), dim3(64), 0, (hipStream_t)stream, a);
    if (d.LK > 0) hipLaunchKernelGGL(attn_dkv_simple, dim3((unsigned)d.LK, (unsigned)d.HKV, (unsigned)d.B), dim3(64), 0, (hipStream_t)stream, a);
    return hip_status(hipGetLastError());
}
