// posit_qk_norm_rope_fwd / posit_qk_norm_rope_bwd: norms of queries and keys for each head with the rotation by positions, and their gradients.
//
// A head's D / 2 pairs go four to a lane: 4 to 32 lanes make a group, which takes one head at a time of a block of rows; a lane keeps its pairs, so weights are decoded once, and the rows'
// cosines and sines are worked out once for all heads (angle in 64 bits, as turns, then its fraction in 32) and shared in LDS.  Queries and keys are a pass each over the block.
#include "heads_common.h"

namespace pnn {

struct Heads {
    const void *x[2], *g[2], *w[2];  // queries, keys
    void *y[2], *dw[2];
    float* rstd_out;
    const float* rstd;
    const int32_t* pos;
    const double* freq;
    uint32_t xl[2], xh[2], gl[2], gh[2];
    int T, H[2], D, R, block;        // block: rows that share a workgroup's angles
    int table;                       // 8-bit posits through a table (forward and backward of 7 rows 19.7 us and 20.3 without, of 4096 51 and 72): 1 of x, 2 of the gradients too, which have x's format
    float eps;
    int kg, kw, ky, kdw;
    ElemFmt fx, fg, fw, fy, fdw;
    float* part;                     // [workgroup][2][D]
};

constexpr int HEADS_BLOCK = 8;

// Cosines and sines of a block of rows into LDS, [row][pair]
__device__ __forceinline__ void heads_angles(const Heads& a, int64_t row0, int rows, float2* cs) {
    const int half = a.R / 2;
    for (int i = threadIdx.x; i < rows * half; i += 256) {
        const int r = i / half, p = i - r * half;
        // as turns, of which only the fraction counts
        double t = (double)a.pos[row0 + r] * a.freq[p] * 0.15915494309189535;
        t -= rint(t);
        float s, c;
        sincospif((float)(2.0 * t), &s, &c);
        cs[r * 128 + p] = make_float2(c, s);
    }
}

__device__ __forceinline__ void heads_pairs(float2 (&cs)[4], const float2* row, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) cs[i] = row[4 * lane + i];
}

// Memory's time would be the least (a head is read and written once); what is longer is the vector unit's: eight elements are looked up, squared, scaled, turned and rounded in some 130
// instructions.  16384 rows of 32 + 8 heads of 128, posit<8,2> to bfloat16: 79 to 85 us.
template <int L, bool NEIGHBOURS, bool WHOLE, int KX>
__global__ __launch_bounds__(256, 4) void heads_fwd_kernel(Heads a) {
    __shared__ float2 angles[HEADS_BLOCK * 128];
    __shared__ uint32_t table[KX == KIND_POSIT_U8 ? 256 * HEADS_COPIES : 1];
    constexpr int GROUPS = 256 / L;
    const int t = threadIdx.x, lane = t % L, group = t / L, heads = a.H[0] + a.H[1];
    const HeadLane<NEIGHBOURS, WHOLE> l(lane, a.D, a.pos ? a.R : 0);
    const bool norm = a.w[0] != nullptr, turn = a.pos != nullptr && a.R > 0, look = KX == KIND_POSIT_U8 && a.table;
    float w[2][8] = {};
    if (norm) {
        heads_weights(w[0], l, a.w[0], a.kw, a.fw);
        if (a.H[1] > 0) heads_weights(w[1], l, a.w[1], a.kw, a.fw);
    }
    if (look) heads_table(table, a.fx);
    const float inv = 1.f / (float)a.D;
    for (int64_t row0 = (int64_t)blockIdx.x * a.block; row0 < a.T; row0 += (int64_t)gridDim.x * a.block) {
        const int rows = a.T - row0 < a.block ? (int)(a.T - row0) : a.block;
        if (turn || look) __syncthreads();
        if (turn) {
            heads_angles(a, row0, rows, angles);
            __syncthreads();
        }
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (a.H[which] == 0) continue;
            const char* const src = (const char*)a.x[which] + row0 * a.xl[which] * (int)sizeof(typename Raw<KX>::T);
            float* const stat = a.rstd_out ? a.rstd_out + row0 * heads + (which ? a.H[0] : 0) : nullptr;
            const int64_t out0 = row0 * a.H[which] * a.D;
            Raw8 next;
            HeadItem it(group, GROUPS, a.H[which]);
            auto load = [&](const HeadItem& i) {
                if (i.r < rows) heads_load(next, l, src, (uint64_t)(uint32_t)i.r * a.xl[which] + (uint64_t)(uint32_t)i.h * a.xh[which], KX);
            };
            load(it);
            while (it.r < rows) {
                const HeadItem at = it;
                float v[8];
                if (look) heads_look_up(v, next, table);
                else values8(v, next, KX, a.fx);
                it.next();
                load(it);
                if (norm) {
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss = fmaf(v[e], v[e], ss);
                    const float rstd = rsqrt_near(fmaf(group_sum<L>(ss), inv, a.eps));
                    if (stat && lane == 0) stat[at.r * heads + at.h] = rstd;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= w[which][e] * rstd;
                }
                if (turn) {
                    float2 cs[4];
                    heads_pairs(cs, angles + at.r * 128, lane);
                    heads_turn<NEIGHBOURS, WHOLE, false>(v, cs, a.R / 2 - 4 * lane);
                }
                Raw8 out;
                raw8<false>(out, v, a.ky, a.fy);
                heads_store(out, l, a.y[which], out0 + (uint32_t)((at.r * a.H[which] + at.h) * a.D), a.ky);
            }
        }
    }
}

// The same bound; dw adds nothing to memory, a lane's pairs being its own: one line a workgroup at the end.  The same sizes: 90 to 101 us.
template <int L, bool NEIGHBOURS, bool WHOLE, int KX>
__global__ __launch_bounds__(256, 4) void heads_bwd_kernel(Heads a) {
    __shared__ float2 angles[HEADS_BLOCK * 128];
    __shared__ uint32_t table[KX == KIND_POSIT_U8 ? 256 * HEADS_COPIES : 1];
    __shared__ float join[256 * 8];
    constexpr int GROUPS = 256 / L;
    const int t = threadIdx.x, lane = t % L, group = t / L, heads = a.H[0] + a.H[1];
    const HeadLane<NEIGHBOURS, WHOLE> l(lane, a.D, a.pos ? a.R : 0);
    const bool norm = a.w[0] != nullptr, turn = a.pos != nullptr && a.R > 0, look = KX == KIND_POSIT_U8 && a.table, look_g = KX == KIND_POSIT_U8 && a.table == 2;
    const int g_bytes = a.kg == KIND_POSIT_U8 ? 1 : (a.kg == KIND_F32 ? 4 : 2);
    float w[2][8] = {}, dw[2][8];
    if (norm) {
        heads_weights(w[0], l, a.w[0], a.kw, a.fw);
        if (a.H[1] > 0) heads_weights(w[1], l, a.w[1], a.kw, a.fw);
    }
    if (look) heads_table(table, a.fx);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[0][e] = dw[1][e] = 0.f;
    const float inv = 1.f / (float)a.D;
    for (int64_t row0 = (int64_t)blockIdx.x * a.block; row0 < a.T; row0 += (int64_t)gridDim.x * a.block) {
        const int rows = a.T - row0 < a.block ? (int)(a.T - row0) : a.block;
        if (turn || look) __syncthreads();
        if (turn) {
            heads_angles(a, row0, rows, angles);
            __syncthreads();
        }
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (a.H[which] == 0) continue;
            const char* const xsrc = (const char*)a.x[which] + (norm ? row0 * a.xl[which] * (int)sizeof(typename Raw<KX>::T) : 0);
            const char* const gsrc = (const char*)a.g[which] + row0 * a.gl[which] * g_bytes;
            const float* const stat = norm ? a.rstd + row0 * heads + (which ? a.H[0] : 0) : nullptr;
            const int64_t out0 = row0 * a.H[which] * a.D;
            Raw8 xr, gr;
            float rs = 0.f;
            HeadItem it(group, GROUPS, a.H[which]);
            auto load = [&](const HeadItem& i) {
                if (i.r >= rows) return;
                heads_load(gr, l, gsrc, (uint64_t)(uint32_t)i.r * a.gl[which] + (uint64_t)(uint32_t)i.h * a.gh[which], a.kg);
                if (norm) {
                    heads_load(xr, l, xsrc, (uint64_t)(uint32_t)i.r * a.xl[which] + (uint64_t)(uint32_t)i.h * a.xh[which], KX);
                    rs = stat[i.r * heads + i.h];
                }
            };
            load(it);
            while (it.r < rows) {
                const HeadItem at = it;
                float g[8], x[8];
                if (look_g) heads_look_up(g, gr, table);
                else values8(g, gr, a.kg, a.fg);
                if (norm) {
                    if (look) heads_look_up(x, xr, table);
                    else values8(x, xr, KX, a.fx);
                }
                const float rstd = rs;
                it.next();
                load(it);
                if (turn) {
                    float2 cs[4];
                    heads_pairs(cs, angles + at.r * 128, lane);
                    heads_turn<NEIGHBOURS, WHOLE, true>(g, cs, a.R / 2 - 4 * lane);
                }
                if (norm) {
                    float c = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x[e] *= rstd;
                        dw[which][e] = fmaf(g[e], x[e], dw[which][e]);
                        g[e] *= w[which][e];
                        c = fmaf(g[e], x[e], c);
                    }
                    c = group_sum<L>(c) * inv;
#pragma unroll
                    for (int e = 0; e < 8; ++e) g[e] = rstd * fmaf(-x[e], c, g[e]);
                }
                Raw8 out;
                raw8<false>(out, g, a.ky, a.fy);
                heads_store(out, l, a.y[which], out0 + (uint32_t)((at.r * a.H[which] + at.h) * a.D), a.ky);
            }
        }
    }
    if (!a.part) return;
    // the groups' sums, in their order, to the workgroup's row (zeros for queries or keys that have no heads)
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) join[e * 256 + t] = dw[which][e];
        __syncthreads();
        for (int i = t; i < 8 * L; i += 256) {
            const int e = i / L, at = i - e * L;
            float s = 0.f;
#pragma unroll
            for (int o = 0; o < GROUPS; ++o) s += join[e * 256 + o * L + at];
            const HeadLane<NEIGHBOURS, WHOLE> lane_of(at, a.D, a.pos ? a.R : 0);
            int first = -1;
#pragma unroll
            for (int y = 0; y < 8; ++y) first = e == y ? lane_of.first(y) : first;
            if (first >= 0) a.part[((int64_t)blockIdx.x * 2 + which) * a.D + first] = s;
        }
    }
}

// The workgroups' sums, 32 columns to a workgroup and 32 runs of rows to each, joined in their order.
__global__ __launch_bounds__(1024) void heads_join_kernel(Heads a, int groups) {
    __shared__ float sums[32][33];
    const int t = threadIdx.x, c = t & 31, run = t >> 5, col = blockIdx.x * 32 + c, cols = 2 * a.D;
    float s = 0.f;
    for (int g0 = run; g0 < groups; g0 += 256) {
        float v[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) v[y] = col < cols && g0 + 32 * y < groups ? a.part[(int64_t)(g0 + 32 * y) * cols + col] : 0.f;
#pragma unroll
        for (int y = 0; y < 8; ++y) s += v[y];
    }
    sums[run][c] = s;
    __syncthreads();
    if (run != 0 || col >= cols) return;
    s = 0.f;
    for (int r = 0; r < 32; ++r) s += sums[r][c];
    const int which = col >= a.D;
    if (a.dw[which]) store_value(a.dw[which], col - (which ? a.D : 0), a.kdw, a.fdw, s);
}

constexpr int64_t HEADS_GROUPS = 1024;

struct HeadsPlan {
    int lanes, block;
    int64_t groups;
};
// Lanes of a head, rows of a block, workgroups: of few rows one each, else as many as the chip holds.
inline HeadsPlan heads_plan(const pnn_heads_desc& d, int64_t most) {
    HeadsPlan p;
    p.lanes = 4;
    while (p.lanes * 8 < d.D) p.lanes *= 2;
    int64_t block = d.T / most;
    p.block = block < 1 ? 1 : (block > HEADS_BLOCK ? HEADS_BLOCK : (int)block);
    p.groups = (d.T + p.block - 1) / p.block;
    if (p.groups > most) p.groups = most;
    return p;
}

inline int heads_status(const pnn_heads_desc* d, bool back) {
    if (!d || d->T < 0 || d->HQ < 0 || d->HKV < 0 || d->D < 0 || d->R < 0 || d->R > d->D || d->R % 2 != 0 || !(d->eps >= 0.f)) return PNN_EINVAL;
    if (d->ql < 0 || d->qh < 0 || d->kl < 0 || d->kh < 0) return PNN_EINVAL;
    if (back && (d->gql < 0 || d->gqh < 0 || d->gkl < 0 || d->gkh < 0)) return PNN_EINVAL;
    for (int64_t stride : {d->ql, d->qh, d->kl, d->kh, back ? d->gql : 0, back ? d->gqh : 0, back ? d->gkl : 0, back ? d->gkh : 0})
        if (stride >= ((int64_t)1 << 32)) return PNN_EUNSUPPORTED;
    if (d->D % 2 != 0 || d->D > 256 || d->T >= ((int64_t)1 << 31) || d->HQ >= 65536 || d->HKV >= 65536 || d->HQ + d->HKV >= 65536) return PNN_EUNSUPPORTED;
    return PNN_OK;
}

template <bool BACK, int KX>
void launch_heads(hipStream_t st, const HeadsPlan& p, bool neighbours, const Heads& a) {
    const dim3 grid((unsigned)p.groups);
#define PNN_HEADS_AS(L, NEIGHBOURS, WHOLE)                                                                                       \
    if (BACK) hipLaunchKernelGGL((heads_bwd_kernel<L, NEIGHBOURS, WHOLE, KX>), grid, dim3(256), 0, st, a);                       \
    else hipLaunchKernelGGL((heads_fwd_kernel<L, NEIGHBOURS, WHOLE, KX>), grid, dim3(256), 0, st, a);
#define PNN_HEADS(L)                        \
    if (neighbours) { PNN_HEADS_AS(L, true, true) } \
    else { PNN_HEADS_AS(L, false, true) }
    if (!heads_whole(a.D, a.pos ? a.R : 0, neighbours)) {
        if (neighbours) { PNN_HEADS_AS(32, true, false) }
        else { PNN_HEADS_AS(32, false, false) }
        return;
    }
    switch (p.lanes) {
        case 4: PNN_HEADS(4) break;
        case 8: PNN_HEADS(8) break;
        case 16: PNN_HEADS(16) break;
        default: PNN_HEADS(32) break;
    }
#undef PNN_HEADS_AS
#undef PNN_HEADS
}

}  // namespace pnn

using namespace pnn;

extern "C" int posit_qk_norm_rope_fwd(void* stream, int fx, int fw, int fy, const pnn_heads_desc* desc, const void* q, const void* k, const void* wq, const void* wk,
                                      const int32_t* pos, const double* inv_freq, void* yq, void* yk, float* rstd) {
    if (const int s = heads_status(desc, false)) return s;
    for (int f : {fx, wq || wk ? fw : fx, fy})
        if (const int s = element_status(f)) return s;
    const pnn_heads_desc& d = *desc;
    if (d.T == 0 || d.HQ + d.HKV == 0 || d.D == 0) return PNN_OK;
    if ((d.HQ > 0 && (!q || !yq)) || (d.HKV > 0 && (!k || !yk)) || (pos && d.R > 0 && !inv_freq)) return PNN_EINVAL;
    const bool norm = wq || wk;
    if (norm && ((d.HQ > 0 && !wq) || (d.HKV > 0 && !wk))) return PNN_EINVAL;
    discard_stale_hip_error();
    const HeadsPlan p = heads_plan(d, HEADS_GROUPS);
    Heads a = {};
    a.x[0] = q; a.x[1] = k; a.y[0] = yq; a.y[1] = yk; a.rstd_out = norm ? rstd : nullptr;
    a.w[0] = norm ? (wq ? wq : wk) : nullptr; a.w[1] = wk;
    a.pos = pos; a.freq = inv_freq;
    a.xl[0] = (uint32_t)d.ql; a.xl[1] = (uint32_t)d.kl; a.xh[0] = (uint32_t)d.qh; a.xh[1] = (uint32_t)d.kh;
    a.T = (int)d.T; a.H[0] = (int)d.HQ; a.H[1] = (int)d.HKV; a.D = (int)d.D; a.R = (int)d.R; a.block = p.block; a.eps = d.eps;
    a.kw = norm ? kind_of(fw) : 0; a.ky = kind_of(fy); a.table = kind_of(fx) == KIND_POSIT_U8;
    a.fx = elem_fmt(fx); a.fw = elem_fmt(norm ? fw : fx); a.fy = elem_fmt(fy);
    PNN_DISPATCH_KIND(kind_of(fx), (launch_heads<false, K>((hipStream_t)stream, p, d.neighbours != 0, a)))
    return hip_status(hipGetLastError());
}

extern "C" size_t posit_qk_norm_rope_bwd_workspace(const pnn_heads_desc* desc) {
    if (heads_status(desc, false) || desc->T == 0 || desc->HQ + desc->HKV == 0 || desc->D == 0) return 0;
    return (size_t)heads_plan(*desc, HEADS_GROUPS).groups * 2 * (size_t)desc->D * 4;
}

extern "C" int posit_qk_norm_rope_bwd(void* stream, int fd, int fx, int fw, int fdx, int fdw, const pnn_heads_desc* desc, const void* dyq, const void* dyk, const void* q,
                                      const void* k, const void* wq, const void* wk, const float* rstd, const int32_t* pos, const double* inv_freq, void* dq, void* dk, void* dwq,
                                      void* dwk, void* workspace, size_t workspace_bytes) {
    if (const int s = heads_status(desc, true)) return s;
    const bool norm = wq || wk, want = norm && (dwq || dwk);
    for (int f : {fd, fx, norm ? fw : fx, fdx, want ? fdw : fx})
        if (const int s = element_status(f)) return s;
    const pnn_heads_desc& d = *desc;
    if (d.T == 0 || d.HQ + d.HKV == 0 || d.D == 0) return PNN_OK;
    if ((d.HQ > 0 && (!dyq || !dq)) || (d.HKV > 0 && (!dyk || !dk)) || (pos && d.R > 0 && !inv_freq)) return PNN_EINVAL;
    if (norm && ((d.HQ > 0 && (!wq || !q)) || (d.HKV > 0 && (!wk || !k)) || !rstd)) return PNN_EINVAL;
    if (!norm && (dwq || dwk)) return PNN_EINVAL;
    const size_t need = want ? posit_qk_norm_rope_bwd_workspace(desc) : 0;
    if (need > 0 && (!workspace || workspace_bytes < need)) return PNN_EWORKSPACE;
    if (need > 0 && !aligned(workspace, 16)) return PNN_EINVAL;
    discard_stale_hip_error();
    const HeadsPlan p = heads_plan(d, HEADS_GROUPS);
    Heads a = {};
    a.x[0] = q; a.x[1] = k; a.g[0] = dyq; a.g[1] = dyk; a.y[0] = dq; a.y[1] = dk; a.dw[0] = dwq; a.dw[1] = dwk; a.rstd = rstd;
    a.w[0] = norm ? (wq ? wq : wk) : nullptr; a.w[1] = wk;
    a.pos = pos; a.freq = inv_freq;
    a.xl[0] = (uint32_t)d.ql; a.xl[1] = (uint32_t)d.kl; a.xh[0] = (uint32_t)d.qh; a.xh[1] = (uint32_t)d.kh;
    a.gl[0] = (uint32_t)d.gql; a.gl[1] = (uint32_t)d.gkl; a.gh[0] = (uint32_t)d.gqh; a.gh[1] = (uint32_t)d.gkh;
    a.T = (int)d.T; a.H[0] = (int)d.HQ; a.H[1] = (int)d.HKV; a.D = (int)d.D; a.R = (int)d.R; a.block = p.block; a.eps = d.eps;
    a.kg = kind_of(fd); a.kw = norm ? kind_of(fw) : 0; a.ky = kind_of(fdx); a.kdw = want ? kind_of(fdw) : 0;
    a.fx = elem_fmt(fx); a.fg = elem_fmt(fd); a.fw = elem_fmt(norm ? fw : fx); a.fy = elem_fmt(fdx); a.fdw = elem_fmt(want ? fdw : fx);
    a.table = kind_of(fx) == KIND_POSIT_U8 ? (fd == fx ? 2 : 1) : 0;
    a.part = want ? (float*)workspace : nullptr;
    hipStream_t st = (hipStream_t)stream;
    PNN_DISPATCH_KIND(kind_of(fx), (launch_heads<true, K>(st, p, d.neighbours != 0, a)))
    if (want) hipLaunchKernelGGL(heads_join_kernel, dim3((unsigned)((2 * d.D + 31) / 32)), dim3(1024), 0, st, a, (int)p.groups);
    return hip_status(hipGetLastError());
}
