// posit_cache_append / posit_cache_read: keys and values into and out of a cache in pages.
//
// What is rounded to a posit or to 4 bits is computed in binary64: then it is the nearest to the formulas' value, however that is computed (in binary32 one value in some 10^7 lies too
// near to a border for that).  Keys and 8-bit queries are a small part of what the vector unit does; queries in bfloat16 and binary32 are computed in binary32, as posit_qk_norm_rope_fwd does.
#include "cache_common.h"

namespace pnn {

struct Append {
    CacheShape s;
    const void *q, *k, *v, *wq, *wk;
    const double* freq;
    char *kc, *vc;
    void* yq;
    uint32_t sl[3], sh[3];   // strides of q, k, v: row, head
    int HQ, R, block, wide;  // wide: queries in binary64
    int table, rounds[2];    // 8-bit posits through a table; rounds of queries and of keys, where workgroups share a block's
    float eps;
    int kw, kq;
    ElemFmt fx, fw, fq, fc;
};

constexpr int APPEND_BLOCK = 8;

// One head's elements: normalised and rotated in T, in the pairs of HeadLane
template <int L, bool NEIGHBOURS, bool WHOLE, class T, class T2>
__device__ __forceinline__ void append_head(T (&x)[8], const float (&v)[8], const Append& a, bool norm, const float (&w)[8], const T2* angles, int lane, int half) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (T)v[e];
    if (norm) {
        T ss = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = __builtin_elementwise_fma(x[e], x[e], ss);
        ss = group_sum<L>(ss) * ((T)1 / (T)a.s.D) + (T)a.eps;
        T rstd;
        if constexpr (sizeof(T) == 8) rstd = rsqrt_wide(ss);
        else rstd = rsqrt_near(ss);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * rstd * (T)w[e];
    }
    if (half) {
        T2 cs[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) cs[i] = angles[4 * lane + i];
        // whole heads without a branch in each lane (the prompts below: 138 us with their reading, 157 with it); lanes behind the head's end turn what nobody stores
        if (2 * half == a.s.D) heads_turn<NEIGHBOURS, WHOLE, false>(x, cs, 4);
        else heads_turn<NEIGHBOURS, WHOLE, false>(x, cs, half - 4 * lane);
    }
}

// A block of rows to a workgroup; 8 or 16 lanes take a head, eight elements to each: of queries and keys four pairs that are rotated, of values and for the cache eight in a row.
// Queries, keys and values are a pass each; of few rows each pass's rounds go to workgroups of their own (gridDim.y).
// Bound by the vector unit, 66 % busy: keys in binary64, conversions of queries.  9 prompts of up to 2048 tokens, 32 + 8 heads of 128, posit<8,2> to bfloat16 and 4 bits: 108 to 112 us, where
// memory would take about 40; 4 tokens 6 us.
template <int L, int KC, int KX, bool NEIGHBOURS, bool WHOLE>
__global__ __launch_bounds__(256, 3) void cache_append_kernel(Append a) {
    __shared__ double2 wide[APPEND_BLOCK * 64];
    __shared__ float2 narrow[APPEND_BLOCK * 64];
    __shared__ float4 rows_of[256 * 2];  // keys on their way from pairs to rows
    __shared__ uint32_t table[KX == KIND_POSIT_U8 ? 256 * HEADS_COPIES : 1];
    __shared__ int seq[APPEND_BLOCK], pos[APPEND_BLOCK];
    constexpr int GROUPS = 256 / L;
    const CacheShape& s = a.s;
    const int t = threadIdx.x, lane = t % L, group = t / L, half = a.freq ? a.R / 2 : 0, D = s.D, d0 = 8 * lane;
    const int left = d0 < D ? 8 : 0;
    const bool look = KX == KIND_POSIT_U8 && a.table;
    const HeadLane<NEIGHBOURS, WHOLE> l(lane, D, half ? a.R : 0);
    float* const mine = (float*)rows_of + group * (L * 8);
    // which passes are this workgroup's, and the first of its groups in them
    const bool alone = gridDim.y == 1;
    const int y = blockIdx.y, only = alone ? -1 : (y < a.rounds[0] ? 0 : (y < a.rounds[0] + a.rounds[1] ? 1 : 2));
    const int round = only <= 0 ? (only == 0 ? y : 0) : (only == 1 ? y - a.rounds[0] : y - a.rounds[0] - a.rounds[1]);
    const int first = round * GROUPS + group, stride = alone ? GROUPS : 1 << 28;
    if (look) heads_table(table, a.fx);
    for (int64_t row0 = (int64_t)blockIdx.x * a.block; row0 < s.T; row0 += (int64_t)gridDim.x * a.block) {
        const int rows = s.T - row0 < a.block ? (int)(s.T - row0) : a.block;
        __syncthreads();
        if (t < APPEND_BLOCK) seq[t] = -1;
        __syncthreads();
        // whose the rows are
        for (int b = t; b < s.B; b += 256) {
            const int begin = cache_first(s, b), end = s.starts ? cache_first(s, b + 1) : b + 1;
            for (int r = 0; r < rows; ++r)
                if (row0 + r >= begin && row0 + r < end) {
                    seq[r] = b;
                    pos[r] = s.lens[b] - (end - (int)(row0 + r));
                }
        }
        __syncthreads();
        if (half)
            for (int i = t; i < rows * half; i += 256) {
                const int r = i / half, p = i - r * half;
                if (seq[r] < 0) continue;
                // as turns, of which only the fraction counts
                double x = (double)pos[r] * a.freq[p] * 0.15915494309189535, sn, cs;
                x -= rint(x);
                sincospi(2.0 * x, &sn, &cs);
                wide[r * 64 + p] = make_double2(cs, sn);
                narrow[r * 64 + p] = make_float2((float)cs, (float)sn);
            }
        __syncthreads();
        // every head of a pass: f(row of the block, head, its elements)
        auto pass = [&](int what, const void* base, int heads, auto f) {
            if (heads == 0 || (only >= 0 && only != what)) return;
            const char* const src = (const char*)base + row0 * a.sl[what] * (int)sizeof(typename Raw<KX>::T);
            Raw8 next;
            next.w = (words8)(0u);
            HeadItem it(first, stride, heads);
            auto load = [&](const HeadItem& i) {
                if (i.r >= rows) return;
                const int64_t at = (uint64_t)(uint32_t)i.r * a.sl[what] + (uint64_t)(uint32_t)i.h * a.sh[what];
                if (what < 2) heads_load(next, l, src, at, KX);
                else if (left) load8(next, src, at + d0, KX, 8);
            };
            load(it);
            while (it.r < rows) {
                const int r = it.r, h = it.h;
                float v[8];
                if (look) heads_look_up(v, next, table);
                else values8(v, next, KX, a.fx);
                it.next();
                load(it);
                if (seq[r] >= 0) f(r, h, v);
            }
        };
        auto put = [&](bool values, int r, int h, float (&v)[8]) {
            const int64_t page = cache_page(s, seq[r], pos[r] >> s.shift, h);
            if (page < 0) return;
            const int at = pos[r] & (s.page - 1);
            char* const to = (values ? a.vc : a.kc) + page;
            if (KC == CACHE_F4) {
                uint32_t most = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t m = bits_of_f32(v[e]) & 0x7FFFFFFFu;
                    most = m > most ? m : most;
                }
                const uint32_t power = f4_power(group_max<4>(left ? most : 0u));
                const uint32_t w = f4_codes(v, power);
                if (left) {
                    *(uint32_t*)(to + cache_unit(s, values, at, lane) / 2) = power == 255u ? 0u : w;
                    if ((lane & 3) == 0) ((uint8_t*)to)[cache_power(s, values, at, lane >> 2)] = (uint8_t)power;
                }
            } else {
                constexpr int K = KC == CACHE_BF16 ? KIND_BF16 : KIND_POSIT_U8;
                Raw8 raw;
                raw8<false>(raw, v, K, a.fc);
                if (left) store8(to, cache_unit(s, values, at, lane), raw, K, 8);
            }
        };
        if (a.q) {
            float w[8] = {};
            if (a.wq && only <= 0) heads_weights(w, l, a.wq, a.kw, a.fw);
            pass(0, a.q, a.HQ, [&](int r, int h, float (&v)[8]) {
                if (a.wide) {
                    double x[8];
                    append_head<L, NEIGHBOURS, WHOLE>(x, v, a, a.wq != nullptr, w, wide + r * 64, lane, half);
                    f32_for_rounding(v, x, a.kq == KIND_POSIT_U8 ? ZEROS_8 : ZEROS_16);
                } else {
                    append_head<L, NEIGHBOURS, WHOLE>(v, v, a, a.wq != nullptr, w, narrow + r * 64, lane, half);
                }
                Raw8 raw;
                raw8<false>(raw, v, a.kq, a.fq);
                heads_store(raw, l, a.yq, ((row0 + r) * a.HQ + h) * D, a.kq);
            });
        }
        if (s.HKV == 0) continue;
        float w[8] = {};
        if (a.wk && (only < 0 || only == 1)) heads_weights(w, l, a.wk, a.kw, a.fw);
        pass(1, a.k, s.HKV, [&](int r, int h, float (&v)[8]) {
            if (a.wk || half) {
                double x[8];
                append_head<L, NEIGHBOURS, WHOLE>(x, v, a, a.wk != nullptr, w, wide + r * 64, lane, half);
                f32_for_rounding(v, x, ZEROS_8);
            }
            // from pairs to rows, inside the wave
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (!WHOLE) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (l.first(e) >= 0) mine[l.first(e)] = v[e];
            } else if (l.in) {
                *(float4*)(mine + l.run0) = make_float4(v[0], v[1], v[2], v[3]);
                *(float4*)(mine + l.run1) = make_float4(v[4], v[5], v[6], v[7]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = mine[d0 + e];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            put(false, r, h, v);
        });
        pass(2, a.v, s.HKV, [&](int r, int h, float (&v)[8]) { put(true, r, h, v); });
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

// Four tokens' eight elements to a thread, of keys or (blockIdx.y) values: a value's four lie side by side.  Bound by the stores: the cache of the prompts above to bfloat16 in 20 us.
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

template <int L, int KC, int KX, bool WHOLE>
void launch_append(hipStream_t st, const dim3& grid, bool neighbours, const Append& a) {
    if (neighbours) hipLaunchKernelGGL((cache_append_kernel<L, KC, KX, true, WHOLE>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((cache_append_kernel<L, KC, KX, false, WHOLE>), grid, dim3(256), 0, st, a);
}
template <int KX>
void launch_append(hipStream_t st, const dim3& grid, int lanes, int kc, bool neighbours, bool whole, const Append& a) {
#define PNN_APPEND(KC)                                                              \
    if (!whole) launch_append<16, KC, KX, false>(st, grid, neighbours, a);          \
    else if (lanes == 8) launch_append<8, KC, KX, true>(st, grid, neighbours, a);   \
    else launch_append<16, KC, KX, true>(st, grid, neighbours, a);
    switch (kc) {
        case CACHE_U8: PNN_APPEND(CACHE_U8) break;
        case CACHE_BF16: PNN_APPEND(CACHE_BF16) break;
        default: PNN_APPEND(CACHE_F4) break;
    }
#undef PNN_APPEND
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
    for (int64_t stride : {q ? d.ql : 0, q ? d.qh : 0, d.kl, d.kh, d.vl, d.vh})
        if (stride >= ((int64_t)1 << 32)) return PNN_EUNSUPPORTED;
    if (!starts && d.T != d.B) return PNN_EINVAL;
    if (d.T == 0 || d.B == 0 || d.D == 0 || (d.HKV == 0 && (d.HQ == 0 || !q))) return PNN_OK;
    if (!lens || (q && !yq) || (norm && ((q && !wq) || !wk))) return PNN_EINVAL;
    if (d.HKV > 0 && (!k || !v || (d.columns > 0 && !table) || (d.pages > 0 && (!k_pages || !v_pages)))) return PNN_EINVAL;
    if (!aligned(k_pages, 16) || !aligned(v_pages, 16)) return PNN_EINVAL;
    Append a = {};
    a.s = cache_shape(d, fcache, starts, lens, table);
    a.q = q; a.k = k; a.v = v; a.wq = wq; a.wk = wk; a.freq = inv_freq; a.kc = (char*)k_pages; a.vc = (char*)v_pages; a.yq = yq;
    a.sl[0] = (uint32_t)d.ql; a.sl[1] = (uint32_t)d.kl; a.sl[2] = (uint32_t)d.vl; a.sh[0] = (uint32_t)d.qh; a.sh[1] = (uint32_t)d.kh; a.sh[2] = (uint32_t)d.vh;
    a.HQ = (int)d.HQ; a.R = (int)d.R; a.wide = q && is_posit(fq); a.eps = d.eps;
    a.kw = norm ? kind_of(fw) : 0; a.kq = q ? kind_of(fq) : 0;
    a.fx = elem_fmt(fx); a.fw = elem_fmt(norm ? fw : fx); a.fq = elem_fmt(q ? fq : fx); a.fc = elem_fmt(fcache);
    const int64_t block = d.T / 512;
    a.block = block < 1 ? 1 : (block > APPEND_BLOCK ? APPEND_BLOCK : (int)block);
    int64_t groups = (d.T + a.block - 1) / a.block;
    if (groups > 65536) groups = 65536;
    const int lanes = !heads_whole(d.D, inv_freq ? d.R : 0, d.neighbours != 0) || d.D > 64 ? 16 : 8;
    // few rows: a round of heads to a workgroup
    const int per = 256 / lanes;
    a.rounds[0] = (int)(((q ? a.block * d.HQ : 0) + per - 1) / per);
    a.rounds[1] = (int)((a.block * d.HKV + per - 1) / per);
    const int64_t rounds = a.rounds[0] + 2 * a.rounds[1];
    const bool share = groups * rounds <= 1024;
    a.table = kind_of(fx) == KIND_POSIT_U8 && !share;  // a workgroup of one round looks up less than it takes to build
    const dim3 grid((unsigned)groups, (unsigned)(share ? rounds : 1));
    hipStream_t st = (hipStream_t)stream;
    discard_stale_hip_error();
    PNN_DISPATCH_KIND(kind_of(fx), (launch_append<K>(st, grid, lanes, cache_kind(fcache), d.neighbours != 0, heads_whole(d.D, inv_freq ? d.R : 0, d.neighbours != 0), a)))
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
