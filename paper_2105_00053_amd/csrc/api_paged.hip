// posit_attention_paged: attention of new tokens over a cache in pages.
#include "attn_paged.h"

namespace pnn {

struct PagedPlan {
    int rows, blocks, tiles, parts;
    int64_t bytes;
};

inline int attn_paged_status(const pnn_paged_desc* d) {
    if (const int s = paged_status(d)) return s;
    if (d->window < 0 || d->sinks < 0 || d->most < 0 || d->longest < 0 || d->ql < 0 || d->qh < 0) return PNN_EINVAL;
    if ((d->HKV == 0) != (d->HQ == 0) || (d->HKV > 0 && d->HQ % d->HKV != 0)) return PNN_EINVAL;
    if (!(d->scale > -3.4028235e38f && d->scale < 3.4028235e38f)) return PNN_EINVAL;
    if (d->longest > ((int64_t)1 << 31) - 128 || (d->HKV > 0 && (d->most > 1024 || d->most * (d->HQ / d->HKV) > 1024))) return PNN_EUNSUPPORTED;
    return PNN_OK;
}

// Keys that any sequence may have
inline int64_t paged_keys(const pnn_paged_desc& d) { return d.longest < d.columns * d.page ? d.longest : d.columns * d.page; }

inline PagedPlan paged_plan(const pnn_paged_desc& d) {
    PagedPlan p = {};
    const int64_t G = d.HQ / d.HKV, longest = paged_keys(d);
    p.rows = d.most * G <= 4 ? 4 : (d.most * G <= 8 ? 8 : 16);
    p.blocks = (int)((d.most * G + p.rows - 1) / p.rows);
    int64_t keys = longest;
    const int64_t window = d.window < longest ? d.window : 0, sinks = d.sinks < longest ? d.sinks : longest;  // both small: their sum is
    if (window > 0 && window + d.most + sinks + 64 < keys) keys = window + d.most + sinks + 64;
    const int64_t all = (keys + 31) / 32 + 1, groups = d.B * d.HKV * p.blocks;
    // three workgroups to a compute unit (64 x 8192 of uneven lengths: 82 us, with two 88; even lengths take 126 with three and 114 with two, but the lengths are not known here)
    int64_t parts = groups > 0 ? (768 + groups - 1) / groups : 1;
    if (parts > all / 4) parts = all / 4;
    if (parts > AT_MOST_PARTS) parts = AT_MOST_PARTS;
    if (parts < 1 || all <= 16) parts = 1;
    p.tiles = (int)((all + parts - 1) / parts);
    p.tiles = (p.tiles + 3) / 4 * 4;
    p.parts = (int)((all + p.tiles - 1) / p.tiles);
    p.bytes = p.parts > 1 ? groups * p.parts * p.rows * (d.D + 2) * 4 : 0;
    return p;
}

template <int KC, int ROWS>
void launch_paged(hipStream_t st, const dim3& grid, const AttnPaged& a) {
    const bool full = a.n.D % 32 == 0;
#define PNN_PAGED(DB)                                                                                              \
    if (full) hipLaunchKernelGGL((attn_paged_kernel<KC, DB, ROWS, true>), grid, dim3(256), 0, st, a);              \
    else hipLaunchKernelGGL((attn_paged_kernel<KC, DB, ROWS, false>), grid, dim3(256), 0, st, a);
    switch ((a.n.D + 31) / 32) {
        case 1: PNN_PAGED(1) break;
        case 2: PNN_PAGED(2) break;
        case 3: PNN_PAGED(3) break;
        default: PNN_PAGED(4) break;
    }
#undef PNN_PAGED
}
template <int KC>
void launch_paged(hipStream_t st, const dim3& grid, const AttnPaged& a) {
    if (a.rows == 4) launch_paged<KC, 4>(st, grid, a);
    else if (a.rows == 8) launch_paged<KC, 8>(st, grid, a);
    else launch_paged<KC, 16>(st, grid, a);
}

}  // namespace pnn

using namespace pnn;

extern "C" size_t posit_attention_paged_workspace(const pnn_paged_desc* desc) {
    if (attn_paged_status(desc) || desc->T == 0 || desc->B == 0 || desc->HQ == 0 || desc->D == 0 || desc->most == 0) return 0;
    return (size_t)paged_plan(*desc).bytes;
}

extern "C" int posit_attention_paged(void* stream, int fq, int fcache, int fout, const pnn_paged_desc* desc, const void* q, const int32_t* starts, const int32_t* lens, const int32_t* table,
                                     const void* k_pages, const void* v_pages, void* o, float* lse, void* workspace, size_t workspace_bytes) {
    if (const int s = attn_paged_status(desc)) return s;
    for (int f : {fq, fout})
        if (const int s = element_status(f)) return s;
    if (fq == PNN_POSIT16_1 || fq == PNN_POSIT12_1 || fq == PNN_F32) return PNN_EUNSUPPORTED;  // more than bfloat16 holds
    if (const int s = cache_format_status(fcache)) return s;
    const pnn_paged_desc& d = *desc;
    if (!starts && d.T != d.B) return PNN_EINVAL;
    if (d.T == 0 || d.B == 0 || d.HQ == 0 || d.D == 0 || d.most == 0) return PNN_OK;
    if (!q || !lens || (d.columns > 0 && !table) || (d.pages > 0 && (!k_pages || !v_pages)) || !o) return PNN_EINVAL;
    if (!aligned(k_pages, 16) || !aligned(v_pages, 16)) return PNN_EINVAL;
    const PagedPlan p = paged_plan(d);
    if ((int64_t)p.blocks * p.parts * d.HKV * d.B > most_workgroups(256) || d.most * (d.HQ / d.HKV) > most_workgroups(512)) return PNN_EUNSUPPORTED;
    if (p.bytes > 0 && (!workspace || workspace_bytes < (size_t)p.bytes)) return PNN_EWORKSPACE;
    if (p.bytes > 0 && !aligned(workspace, 16)) return PNN_EINVAL;
    AttnPaged a = {};
    a.s = cache_shape(d, fcache, starts, lens, table);
    const int64_t keys = paged_keys(d);
    a.n.LK = (int)keys;
    a.n.window = d.window >= keys ? 0 : (int)d.window;  // a window of all keys is none
    a.n.sinks = (int)(d.sinks < keys ? d.sinks : keys);
    a.n.HKV = (int)d.HKV; a.n.G = (int)(d.HQ / d.HKV); a.n.D = (int)d.D; a.n.scale = d.scale;
    a.q = q; a.k = (const char*)k_pages; a.v = (const char*)v_pages; a.ql = d.ql; a.qh = d.qh; a.kq = kind_of(fq); a.most = (int)d.most; a.fq = elem_fmt(fq); a.fc = elem_fmt(fcache);
    a.o = o; a.lse = lse; a.ko = kind_of(fout); a.fo = elem_fmt(fout);
    a.rows = p.rows; a.blocks = p.blocks; a.tiles = p.tiles; a.parts = p.parts; a.part = (float*)workspace;
    hipStream_t st = (hipStream_t)stream;
    discard_stale_hip_error();
    if (d.pages == 0) {
        hipLaunchKernelGGL(attn_paged_none_kernel, dim3((unsigned)d.most, (unsigned)d.B), dim3(256), 0, st, a);
        return hip_status(hipGetLastError());
    }
    const dim3 grid((unsigned)((int64_t)p.blocks * p.parts * d.HKV * d.B));
    switch (cache_kind(fcache)) {
        case CACHE_U8: launch_paged<CACHE_U8>(st, grid, a); break;
        case CACHE_BF16: launch_paged<CACHE_BF16>(st, grid, a); break;
        default: launch_paged<CACHE_F4>(st, grid, a); break;
    }
    if (p.parts > 1) hipLaunchKernelGGL(attn_paged_join_kernel, dim3((unsigned)(d.most * a.n.G), (unsigned)d.HKV, (unsigned)d.B), dim3(512), 0, st, a);
    return hip_status(hipGetLastError());
}
