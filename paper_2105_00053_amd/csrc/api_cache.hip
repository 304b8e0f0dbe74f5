// posit_cache_append / posit_cache_read: keys and values into and out of a cache in pages.
//
// Append computes in binary64: a stored element is the nearest to the formulas' value, whichever way that is computed, and what it costs is hidden behind the memory (the
// vector unit's binary64 rate is that of binary32).
#include "cache_common.h"

namespace pnn {

struct Append {
    CacheShape s;
    const void *q, *k, *v, *wq, *wk;
    const double* freq;
    char *kc, *vc;
    void* yq;
    int64_t ql, qh, kl, kh, vl, vh;
    int HQ, R, neighbours, block;
    double eps;
    int kx, kw, kq;
    ElemFmt fx, fw, fq, fc;
};

constexpr int APPEND_BLOCK = 4;

// A block of rows to a workgroup (of which gridDim.y share its heads); 4, 8 or 16 lanes take a head, eight elements in a row to each.
template <int L, int KC>
__global__ __launch_bounds__(256) void cache_append_kernel(Append a) {
    __shared__ double2 angles[APPEND_BLOCK * 64];
    __shared__ double heads[256 * 8];
    __shared__ int seq[APPEND_BLOCK], pos[APPEND_BLOCK];
    constexpr int GROUPS = 256 / L;
    const CacheShape& s = a.s;
    const int t = threadIdx.x, lane = t % L, group = t / L, half = a.freq ? a.R / 2 : 0, D = s.D, d0 = 8 * lane;
    const int left = D - d0 < 0 ? 0 : (D - d0 < 8 ? D - d0 : 8);
    const int hq = a.q ? a.HQ : 0, all = hq + 2 * s.HKV;
    double* const mine = heads + group * (L * 8);
    for (int64_t row0 = (int64_t)blockIdx.x * a.block; row0 < s.T; row0 += (int64_t)gridDim.x * a.block) {
        const int rows = s.T - row0 < a.block ? (int)(s.T - row0) : a.block;
        __syncthreads();
        if (t < APPEND_BLOCK) seq[t] = -1;
        __syncthreads();
        // whose the rows are
        for (int b = t; b < s.B; b += 256) {
            const int first = cache_first(s, b), end = s.starts ? cache_first(s, b + 1) : b + 1;
            for (int r = 0; r < rows; ++r)
                if (row0 + r >= first && row0 + r < end) {
                    seq[r] = b;
                    pos[r] = s.lens[b] - (end - (int)(row0 + r));
                }
        }
        __syncthreads();
        for (int i = t; i < rows * half; i += 256) {
            const int r = i / half, p = i - r * half;
            if (seq[r] < 0) continue;
            // as turns, of which only the fraction counts
            double x = (double)pos[r] * a.freq[p] * 0.15915494309189535, sn, cs;
            x -= rint(x);
            sincospi(2.0 * x, &sn, &cs);
            angles[i] = make_double2(cs, sn);
        }
        __syncthreads();
        for (int item = blockIdx.y * GROUPS + group; item < rows * all; item += GROUPS * gridDim.y) {
            const int r = item / all, n = item - r * all, b = seq[r];
            if (b < 0) continue;
            const int what = n < hq ? 0 : (n < hq + s.HKV ? 1 : 2), h = what == 0 ? n : (n - hq) - (what == 2 ? s.HKV : 0);
            const int64_t row = row0 + r;
            const int at = pos[r] & (s.page - 1);
            int64_t page = 0;
            if (what) {
                page = cache_page(s, b, pos[r] >> s.shift, h);
                if (page < 0) continue;
            }
            Raw8 raw;
            const void* const src = what == 0 ? a.q : (what == 1 ? a.k : a.v);
            load8(raw, src, row * (what == 0 ? a.ql : (what == 1 ? a.kl : a.vl)) + h * (what == 0 ? a.qh : (what == 1 ? a.kh : a.vh)) + d0, a.kx, left);
            float v[8];
            values8(v, raw, a.kx, a.fx);
            if (what != 2 && (a.wk || half)) {
                double x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = e < left ? (double)v[e] : 0.0;
                if (a.wk) {
                    double ss = 0.0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss = fma(x[e], x[e], ss);
                    const double rstd = 1.0 / sqrt(group_sum<L>(ss) / D + a.eps);
                    Raw8 wr;
                    float w[8];
                    load8(wr, what ? a.wk : a.wq, d0, a.kw, left);
                    values8(w, wr, a.kw, a.fw);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = x[e] * rstd * (double)w[e];
                }
                if (half) {
                    // each element's other one through LDS, inside the wave
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                    for (int e = 0; e < 8; ++e) mine[d0 + e] = x[e];
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int d = d0 + e;
                        if (d >= 2 * half) continue;
                        const int p = a.neighbours ? d >> 1 : (d < half ? d : d - half);
                        const bool second = a.neighbours ? d & 1 : d >= half;
                        const double2 cs = angles[r * half + p];
                        const double other = mine[a.neighbours ? d ^ 1 : (second ? d - half : d + half)];
                        x[e] = fma(x[e], cs.x, (second ? other : -other) * cs.y);
                    }
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = what == 0 && a.kq == KIND_F32 ? (float)x[e] : f32_to_odd(x[e]);
            }
            if (what == 0) {
                raw8<false>(raw, v, a.kq, a.fq);
                store8(a.yq, (row * a.HQ + h) * D + d0, raw, a.kq, left);
                continue;
            }
            const bool values = what == 2;
            char* const to = (values ? a.vc : a.kc) + page;
            if (KC == CACHE_F4) {
                uint32_t most = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t m = e < left ? bits_of_f32(v[e]) & 0x7FFFFFFFu : 0u;
                    most = m > most ? m : most;
                }
                const uint32_t power = f4_power(group_max<4>(most));
                const float inverse = f32_of_bits((254u - power) << 23);
                uint32_t w = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) w |= f4_code(v[e], inverse) << (4 * e);
                if (left) {
                    *(uint32_t*)(to + cache_unit(s, values, at, lane) / 2) = power == 255u ? 0u : w;
                    if ((lane & 3) == 0) ((uint8_t*)to)[cache_power(s, values, at, lane >> 2)] = (uint8_t)power;
                }
            } else {
                constexpr int K = KC == CACHE_BF16 ? KIND_BF16 : KIND_POSIT_U8;
                raw8<false>(raw, v, K, a.fc);
                if (left) store8(to, cache_unit(s, values, at, lane), raw, K, 8);
            }
        }
    }
}

struct CacheRead {
    CacheShape s;
    const char *kc, *vc;
    void *k, *v;
    int64_t longest, items;
    int kout;
    ElemFmt fc, fout;
};

// Four tokens' eight elements to a thread, of keys or (blockIdx.y) values: a value's four lie side by side.
template <int KC>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheRead a) {
    const CacheShape& s = a.s;
    const bool values = blockIdx.y != 0;
    const int units = s.D >> 3, quads = (int)((a.longest + 3) / 4);
    for (int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x; item < a.items; item += (int64_t)gridDim.x * 256) {
        const int unit = (int)(item % units);
        const int64_t x = item / units, y = x / s.HKV;
        const int h = (int)(x - y * s.HKV), b = (int)(y / quads), j = (int)(y - (int64_t)b * quads) * 4;
        const int keys = s.lens[b] < a.longest ? s.lens[b] : (int)a.longest;
        const int64_t page = j < keys ? cache_page(s, b, j >> s.shift, h) : -1;
        const char* const from = (values ? a.vc : a.kc) + page;
        const int at = j & (s.page - 1);
        float v[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = j + i < keys ? f32_of_bits(0x7FC00000u) : 0.f;
            if (page < 0 || j + i >= keys) continue;
            const int el = cache_unit(s, values, at + i, unit);
            if (KC == CACHE_F4) {
                f4_values(v[i], *(const uint32_t*)(from + el / 2), ((const uint8_t*)from)[cache_power(s, values, at + i, unit >> 2)]);
            } else {
                constexpr int K = KC == CACHE_BF16 ? KIND_BF16 : KIND_POSIT_U8;
                Raw8 raw;
                load8(raw, from, el, K, 8);
                values8(v[i], raw, K, a.fc);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (j + i >= a.longest) break;
            Raw8 raw;
            raw8<false>(raw, v[i], a.kout, a.fout);
            store8(values ? a.v : a.k, (((int64_t)b * a.longest + j + i) * s.HKV + h) * s.D + unit * 8, raw, a.kout, 8);
        }
    }
}

}  // namespace pnn

using namespace pnn;

extern "C" int posit_cache_append(void* stream, int fx, int fw, int fq, int fcache, const pnn_paged_desc* desc, const void* q, const void* k, const void* v, const void* wq, const void* wk,
                                  const double* inv_freq, const int32_t* starts, const int32_t* lens, const int32_t* table, void* k_pages, void* v_pages, void* yq) {
    if (const int s = paged_status(desc)) return s;
    const pnn_paged_desc& d = *desc;
    if (d.R < 0 || d.R > d.D || d.R % 2 != 0 || !(d.eps >= 0.f) || (q && (d.ql < 0 || d.qh < 0)) || d.kl < 0 || d.kh < 0 || d.vl < 0 || d.vh < 0) return PNN_EINVAL;
    const bool norm = wq || wk;
    for (int f : {fx, norm ? fw : fx, q ? fq : fx})
        if (const int s = element_status(f)) return s;
    if (const int s = cache_format_status(fcache)) return s;
    if (!starts && d.T != d.B) return PNN_EINVAL;
    if (d.T == 0 || d.B == 0 || d.D == 0 || (d.HKV == 0 && (d.HQ == 0 || !q))) return PNN_OK;
    if (!lens || (q && !yq) || (norm && ((q && !wq) || !wk))) return PNN_EINVAL;
    if (d.HKV > 0 && (!k || !v || (d.columns > 0 && !table) || (d.pages > 0 && (!k_pages || !v_pages)))) return PNN_EINVAL;
    if (!aligned(k_pages, 16) || !aligned(v_pages, 16)) return PNN_EINVAL;
    Append a = {};
    a.s = cache_shape(d, fcache, starts, lens, table);
    a.q = q; a.k = k; a.v = v; a.wq = wq; a.wk = wk; a.freq = inv_freq; a.kc = (char*)k_pages; a.vc = (char*)v_pages; a.yq = yq;
    a.ql = d.ql; a.qh = d.qh; a.kl = d.kl; a.kh = d.kh; a.vl = d.vl; a.vh = d.vh;
    a.HQ = (int)d.HQ; a.R = (int)d.R; a.neighbours = d.neighbours != 0; a.eps = d.eps;
    a.kx = kind_of(fx); a.kw = norm ? kind_of(fw) : 0; a.kq = q ? kind_of(fq) : 0;
    a.fx = elem_fmt(fx); a.fw = elem_fmt(norm ? fw : fx); a.fq = elem_fmt(q ? fq : fx); a.fc = elem_fmt(fcache);
    const int64_t block = d.T / 2048;
    a.block = block < 1 ? 1 : (block > APPEND_BLOCK ? APPEND_BLOCK : (int)block);
    int64_t groups = (d.T + a.block - 1) / a.block;
    if (groups > 65536) groups = 65536;
    const int lanes = d.D <= 32 ? 4 : (d.D <= 64 ? 8 : 16);
    // few rows: a row's heads shared out, so that a group of lanes takes one
    const int64_t items = a.block * ((q ? d.HQ : 0) + 2 * d.HKV), rounds = (items * lanes + 255) / 256;
    const int64_t shares = groups * rounds <= 1024 ? rounds : 1;
    const dim3 grid((unsigned)groups, (unsigned)(shares < 65536 ? shares : 65535));
    hipStream_t st = (hipStream_t)stream;
    discard_stale_hip_error();
#define PNN_APPEND(L)                                                                                          \
    switch (cache_kind(fcache)) {                                                                              \
        case CACHE_U8: hipLaunchKernelGGL((cache_append_kernel<L, CACHE_U8>), grid, dim3(256), 0, st, a); break;     \
        case CACHE_BF16: hipLaunchKernelGGL((cache_append_kernel<L, CACHE_BF16>), grid, dim3(256), 0, st, a); break; \
        default: hipLaunchKernelGGL((cache_append_kernel<L, CACHE_F4>), grid, dim3(256), 0, st, a); break;           \
    }
    if (lanes == 4) { PNN_APPEND(4) }
    else if (lanes == 8) { PNN_APPEND(8) }
    else { PNN_APPEND(16) }
#undef PNN_APPEND
    return hip_status(hipGetLastError());
}

extern "C" int posit_cache_read(void* stream, int fcache, int fout, const pnn_paged_desc* desc, const int32_t* lens, const int32_t* table, const void* k_pages, const void* v_pages, void* k, void* v) {
    if (const int s = paged_status(desc)) return s;
    const pnn_paged_desc& d = *desc;
    if (d.longest < 0) return PNN_EINVAL;
    if (d.longest >= ((int64_t)1 << 31) - 128) return PNN_EUNSUPPORTED;
    if (const int s = cache_format_status(fcache)) return s;
    if (const int s = element_status(fout)) return s;
    if (d.B == 0 || d.HKV == 0 || d.D == 0 || d.longest == 0) return PNN_OK;
    if (!lens || (d.columns > 0 && !table) || (d.pages > 0 && (!k_pages || !v_pages)) || !k || !v) return PNN_EINVAL;
    if (!aligned(k_pages, 16) || !aligned(v_pages, 16)) return PNN_EINVAL;
    CacheRead a = {};
    a.s = cache_shape(d, fcache, nullptr, lens, table);
    a.kc = (const char*)k_pages; a.vc = (const char*)v_pages; a.k = k; a.v = v;
    a.longest = d.longest; a.items = d.B * ((d.longest + 3) / 4) * d.HKV * (d.D / 8);
    a.kout = kind_of(fout); a.fc = elem_fmt(fcache); a.fout = elem_fmt(fout);
    int64_t groups = (a.items + 255) / 256;
    if (groups > 65536) groups = 65536;
    hipStream_t st = (hipStream_t)stream;
    discard_stale_hip_error();
    const dim3 grid((unsigned)groups, 2);
    switch (cache_kind(fcache)) {
        case CACHE_U8: hipLaunchKernelGGL(cache_read_kernel<CACHE_U8>, grid, dim3(256), 0, st, a); break;
        case CACHE_BF16: hipLaunchKernelGGL(cache_read_kernel<CACHE_BF16>, grid, dim3(256), 0, st, a); break;
        default: hipLaunchKernelGGL(cache_read_kernel<CACHE_F4>, grid, dim3(256), 0, st, a); break;
    }
    return hip_status(hipGetLastError());
}
