// posit_qk_norm_rope_fwd / posit_qk_norm_rope_bwd: norms of queries and keys for each head with the rotation by positions, and their gradients.
//
// A head's D / 2 pairs go four to a lane: 8, 16 or 32 elements' lanes make a group, which takes one head at a time of a block of rows; a lane keeps its pairs, so weights are decoded
// once, and the rows' cosines and sines are worked out once for all heads (angle in 64 bits, as turns, then its fraction in 32) and shared in LDS.
#include "heads_common.h"

namespace pnn {

struct Heads {
    const void *x[2], *g[2], *w[2];  // queries, keys
    void *y[2], *dw[2];
    float* rstd_out;
    const float* rstd;
    const int32_t* pos;
    const double* freq;
    int64_t xl[2], xh[2], gl[2], gh[2];
    int T, H[2], D, R, block;        // block: rows that share a workgroup's angles
    float eps;
    int kx, kg, kw, ky, kdw;
    ElemFmt fx, fg, fw, fy, fdw;
    float* part;                     // [workgroup][2][D]
};

constexpr int HEADS_BLOCK = 8;

// Cosines and sines of a block of rows into LDS: [row][R / 2]
__device__ __forceinline__ void heads_angles(const Heads& a, int row0, int rows, float2* cs) {
    const int half = a.R / 2;
    for (int i = threadIdx.x; i < rows * half; i += 256) {
        const int r = i / half, p = i - r * half;
        // as turns, of which only the fraction counts
        double t = (double)a.pos[row0 + r] * a.freq[p] * 0.15915494309189535;
        t -= rint(t);
        float s, c;
        sincospif((float)(2.0 * t), &s, &c);
        cs[i] = make_float2(c, s);
    }
}

// A lane's elements: 0 .. 3 the firsts of its four pairs and 4 .. 7 the seconds, or, of neighbours, as they lie.  WHOLE: both runs of four are inside
// a head and on one side of R / 2.
template <bool NEIGHBOURS>
struct HeadLane {
    int first[8];  // element of the head, or -1
    bool whole;
    int run0, run1;
    __device__ __forceinline__ HeadLane(int lane, int D, int R) {
        const int half = R / 2, rest = (D - R) / 2;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int p = 4 * lane + (NEIGHBOURS ? e / 2 : e & 3), second = NEIGHBOURS ? e & 1 : e >> 2;
            if (NEIGHBOURS) first[e] = 2 * p + second;
            else first[e] = p < half ? p + second * half : R + (p - half) + second * rest;
            if (p >= D / 2) first[e] = -1;
        }
        run0 = first[0];
        run1 = first[4];
        whole = first[0] >= 0 && first[7] >= 0 && first[3] == run0 + 3 && first[7] == run1 + 3;
    }
};

template <bool NEIGHBOURS>
__device__ __forceinline__ void heads_load(Raw8& r, const HeadLane<NEIGHBOURS>& l, const void* p, int64_t at, int kind) {
    if (l.whole) {
        if (NEIGHBOURS) {
            load8(r, p, at + l.run0, kind, 8);
        } else if (kind == KIND_POSIT_U8) {
            uint32_t b[2];
            __builtin_memcpy(&b[0], (const uint8_t*)p + at + l.run0, 4);
            __builtin_memcpy(&b[1], (const uint8_t*)p + at + l.run1, 4);
            r.w[0] = b[0];
            r.w[1] = b[1];
        } else if (kind == KIND_F32) {
            r.w.lo = *(const words4_any*)((const uint32_t*)p + at + l.run0);
            r.w.hi = *(const words4_any*)((const uint32_t*)p + at + l.run1);
        } else {
            r.w.lo.lo = *(const words2_any*)((const uint16_t*)p + at + l.run0);
            r.w.lo.hi = *(const words2_any*)((const uint16_t*)p + at + l.run1);
        }
        return;
    }
    r.w = (words8)(0u);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (l.first[e] < 0) continue;
        const int64_t i = at + l.first[e];
        if (kind == KIND_POSIT_U8) r.w[e / 4] |= (uint32_t)((const uint8_t*)p)[i] << (8 * (e & 3));
        else if (kind == KIND_F32) r.w[e] = ((const uint32_t*)p)[i];
        else r.w[e / 2] |= (uint32_t)((const uint16_t*)p)[i] << (16 * (e & 1));
    }
}

template <bool NEIGHBOURS>
__device__ __forceinline__ void heads_store(const Raw8& r, const HeadLane<NEIGHBOURS>& l, void* p, int64_t at, int kind) {
    if (l.whole) {
        if (NEIGHBOURS) {
            store8(p, at + l.run0, r, kind, 8);
        } else if (kind == KIND_POSIT_U8) {
            const uint32_t b[2] = {r.w[0], r.w[1]};
            __builtin_memcpy((uint8_t*)p + at + l.run0, &b[0], 4);
            __builtin_memcpy((uint8_t*)p + at + l.run1, &b[1], 4);
        } else if (kind == KIND_F32) {
            *(words4_any*)((uint32_t*)p + at + l.run0) = r.w.lo;
            *(words4_any*)((uint32_t*)p + at + l.run1) = r.w.hi;
        } else {
            *(words2_any*)((uint16_t*)p + at + l.run0) = r.w.lo.lo;
            *(words2_any*)((uint16_t*)p + at + l.run1) = r.w.lo.hi;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (l.first[e] < 0) continue;
        const int64_t i = at + l.first[e];
        if (kind == KIND_POSIT_U8) ((uint8_t*)p)[i] = (uint8_t)(r.w[e / 4] >> (8 * (e & 3)));
        else if (kind == KIND_F32) ((uint32_t*)p)[i] = r.w[e];
        else ((uint16_t*)p)[i] = (uint16_t)(r.w[e / 2] >> (16 * (e & 1)));
    }
}

// The lane's pairs by its angles; BACK: by their negatives
template <bool NEIGHBOURS, bool BACK>
__device__ __forceinline__ void heads_turn(float (&v)[8], const float2 (&cs)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        constexpr int step = NEIGHBOURS ? 2 : 1, gap = NEIGHBOURS ? 1 : 4;
        const int x = step * i, y = x + gap;
        const float s = BACK ? -cs[i].y : cs[i].y, a = v[x], b = v[y];
        v[x] = fmaf(a, cs[i].x, -(b * s));
        v[y] = fmaf(b, cs[i].x, a * s);
    }
}

template <bool NEIGHBOURS>
__device__ __forceinline__ void heads_weights(float (&w)[8], const Heads& a, const HeadLane<NEIGHBOURS>& l, int which) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = l.first[e] >= 0 ? load_value(a.w[which], l.first[e], a.kw, a.fw) : 0.f;
}

template <int L, bool NEIGHBOURS, int KX>
__global__ __launch_bounds__(256) void heads_fwd_kernel(Heads a) {
    __shared__ float2 angles[HEADS_BLOCK * 128];
    constexpr int GROUPS = 256 / L;
    const int t = threadIdx.x, lane = t % L, group = t / L, heads = a.H[0] + a.H[1], half = a.R / 2;
    const HeadLane<NEIGHBOURS> l(lane, a.D, a.R);
    const bool norm = a.w[0] != nullptr, turn = a.pos != nullptr && half > 0;
    float w[2][8];
    if (norm) {
        heads_weights(w[0], a, l, 0);
        if (a.H[1] > 0) heads_weights(w[1], a, l, 1);
    }
    const float inv = 1.f / (float)a.D;
    for (int64_t row0 = (int64_t)blockIdx.x * a.block; row0 < a.T; row0 += (int64_t)gridDim.x * a.block) {
        const int rows = a.T - row0 < a.block ? (int)(a.T - row0) : a.block, items = rows * heads;
        if (turn) {
            __syncthreads();
            heads_angles(a, (int)row0, rows, angles);
            __syncthreads();
        }
        Raw8 next;
        auto load = [&](int item) {
            const int r = item / heads, h = item - r * heads, which = h >= a.H[0];
            heads_load(next, l, a.x[which], (row0 + r) * a.xl[which] + (h - (which ? a.H[0] : 0)) * a.xh[which], KX);
        };
        if (group < items) load(group);
        for (int item = group; item < items; item += GROUPS) {
            const int r = item / heads, h = item - r * heads, which = h >= a.H[0];
            float v[8];
            values8(v, next, KX, a.fx);
            if (item + GROUPS < items) load(item + GROUPS);
            const int64_t row = row0 + r;
            if (norm) {
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(v[e], v[e], ss);
                const float rstd = 1.f / sqrtf(group_sum<L>(ss) * inv + a.eps);
                if (a.rstd_out && lane == 0) a.rstd_out[row * heads + h] = rstd;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= (which ? w[1][e] : w[0][e]) * rstd;
            }
            if (turn) {
                float2 cs[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) cs[i] = 4 * lane + i < half ? angles[r * half + 4 * lane + i] : make_float2(1.f, 0.f);
                heads_turn<NEIGHBOURS, false>(v, cs);
            }
            Raw8 out;
            raw8<false>(out, v, a.ky, a.fy);
            heads_store(out, l, a.y[which], (row * a.H[which] + (h - (which ? a.H[0] : 0))) * a.D, a.ky);
        }
    }
}

template <int L, bool NEIGHBOURS, int KX>
__global__ __launch_bounds__(256) void heads_bwd_kernel(Heads a) {
    __shared__ float2 angles[HEADS_BLOCK * 128];
    __shared__ float join[256 * 8];
    constexpr int GROUPS = 256 / L;
    const int t = threadIdx.x, lane = t % L, group = t / L, heads = a.H[0] + a.H[1], half = a.R / 2;
    const HeadLane<NEIGHBOURS> l(lane, a.D, a.R);
    const bool norm = a.w[0] != nullptr, turn = a.pos != nullptr && half > 0;
    float w[2][8], dw[2][8];
    if (norm) {
        heads_weights(w[0], a, l, 0);
        if (a.H[1] > 0) heads_weights(w[1], a, l, 1);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[0][e] = dw[1][e] = 0.f;
    const float inv = 1.f / (float)a.D;
    for (int64_t row0 = (int64_t)blockIdx.x * a.block; row0 < a.T; row0 += (int64_t)gridDim.x * a.block) {
        const int rows = a.T - row0 < a.block ? (int)(a.T - row0) : a.block, items = rows * heads;
        if (turn) {
            __syncthreads();
            heads_angles(a, (int)row0, rows, angles);
            __syncthreads();
        }
        Raw8 xr, gr;
        float rs = 0.f;
        auto load = [&](int item) {
            const int r = item / heads, h = item - r * heads, which = h >= a.H[0], hh = h - (which ? a.H[0] : 0);
            heads_load(gr, l, a.g[which], (row0 + r) * a.gl[which] + hh * a.gh[which], a.kg);
            if (norm) {
                heads_load(xr, l, a.x[which], (row0 + r) * a.xl[which] + hh * a.xh[which], KX);
                rs = a.rstd[(row0 + r) * heads + h];
            }
        };
        if (group < items) load(group);
        for (int item = group; item < items; item += GROUPS) {
            const int r = item / heads, h = item - r * heads, which = h >= a.H[0];
            float g[8], x[8];
            values8(g, gr, a.kg, a.fg);
            if (norm) values8(x, xr, KX, a.fx);
            const float rstd = rs;
            if (item + GROUPS < items) load(item + GROUPS);
            if (turn) {
                float2 cs[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) cs[i] = 4 * lane + i < half ? angles[r * half + 4 * lane + i] : make_float2(1.f, 0.f);
                heads_turn<NEIGHBOURS, true>(g, cs);
            }
            if (norm) {
                float c = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] *= rstd;
                    const float d = g[e] * x[e];
                    if (which) dw[1][e] += d;
                    else dw[0][e] += d;
                    g[e] *= which ? w[1][e] : w[0][e];
                    c = fmaf(g[e], x[e], c);
                }
                c = group_sum<L>(c) * inv;
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] = rstd * fmaf(-x[e], c, g[e]);
            }
            Raw8 out;
            raw8<false>(out, g, a.ky, a.fy);
            heads_store(out, l, a.y[which], ((row0 + r) * a.H[which] + (h - (which ? a.H[0] : 0))) * a.D, a.ky);
        }
    }
    if (!a.part) return;
    // the groups' sums, in their order, to the workgroup's row
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) join[t * 8 + e] = which ? dw[1][e] : dw[0][e];
        __syncthreads();
        if (t < L)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float s = 0.f;
                for (int o = 0; o < GROUPS; ++o) s += join[(o * L + t) * 8 + e];
                if (l.first[e] >= 0) a.part[((int64_t)blockIdx.x * 2 + which) * a.D + l.first[e]] = s;
            }
    }
}

// The workgroups' sums, 8 columns to a workgroup and 32 runs of rows to each, joined in their order.
__global__ __launch_bounds__(256) void heads_join_kernel(Heads a, int groups) {
    __shared__ float sums[32][9];
    const int t = threadIdx.x, c = t & 7, run = t >> 3, col = blockIdx.x * 8 + c;
    float s = 0.f;
    if (col < 2 * a.D)
        for (int g = run; g < groups; g += 32) s += a.part[(int64_t)g * 2 * a.D + col];
    sums[run][c] = s;
    __syncthreads();
    if (run != 0 || col >= 2 * a.D) return;
    s = 0.f;
    for (int r = 0; r < 32; ++r) s += sums[r][c];
    const int which = col >= a.D;
    if (a.dw[which]) store_value(a.dw[which], col - (which ? a.D : 0), a.kdw, a.fdw, s);
}

constexpr int64_t HEADS_GROUPS = 2048;

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
    if (d->D % 2 != 0 || d->D > 256 || d->T >= ((int64_t)1 << 31) || d->HQ >= 65536 || d->HKV >= 65536 || d->HQ + d->HKV >= 65536) return PNN_EUNSUPPORTED;
    return PNN_OK;
}

template <bool BACK, int KX>
void launch_heads(hipStream_t st, const HeadsPlan& p, bool neighbours, const Heads& a) {
    const dim3 grid((unsigned)p.groups);
#define PNN_HEADS(L)                                                                                                              \
    if (BACK) {                                                                                                                    \
        if (neighbours) hipLaunchKernelGGL((heads_bwd_kernel<L, true, KX>), grid, dim3(256), 0, st, a);                            \
        else hipLaunchKernelGGL((heads_bwd_kernel<L, false, KX>), grid, dim3(256), 0, st, a);                                      \
    } else {                                                                                                                       \
        if (neighbours) hipLaunchKernelGGL((heads_fwd_kernel<L, true, KX>), grid, dim3(256), 0, st, a);                            \
        else hipLaunchKernelGGL((heads_fwd_kernel<L, false, KX>), grid, dim3(256), 0, st, a);                                      \
    }
    switch (p.lanes) {
        case 4: PNN_HEADS(4) break;
        case 8: PNN_HEADS(8) break;
        case 16: PNN_HEADS(16) break;
        default: PNN_HEADS(32) break;
    }
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
    a.xl[0] = d.ql; a.xl[1] = d.kl; a.xh[0] = d.qh; a.xh[1] = d.kh;
    a.T = (int)d.T; a.H[0] = (int)d.HQ; a.H[1] = (int)d.HKV; a.D = (int)d.D; a.R = (int)d.R; a.block = p.block; a.eps = d.eps;
    a.kx = kind_of(fx); a.kw = norm ? kind_of(fw) : 0; a.ky = kind_of(fy);
    a.fx = elem_fmt(fx); a.fw = elem_fmt(norm ? fw : fx); a.fy = elem_fmt(fy);
    PNN_DISPATCH_KIND(a.kx, (launch_heads<false, K>((hipStream_t)stream, p, d.neighbours != 0, a)))
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
    a.x[0] = q; a.x[1] = k; a.g[0] = dyq; a.g[1] = dyk; a.y[0] = dq; a.y[1] = dk; a.dw[0] = d.HQ > 0 ? dwq : nullptr; a.dw[1] = d.HKV > 0 ? dwk : nullptr; a.rstd = rstd;
    a.w[0] = norm ? (wq ? wq : wk) : nullptr; a.w[1] = wk;
    a.pos = pos; a.freq = inv_freq;
    a.xl[0] = d.ql; a.xl[1] = d.kl; a.xh[0] = d.qh; a.xh[1] = d.kh;
    a.gl[0] = d.gql; a.gl[1] = d.gkl; a.gh[0] = d.gqh; a.gh[1] = d.gkh;
    a.T = (int)d.T; a.H[0] = (int)d.HQ; a.H[1] = (int)d.HKV; a.D = (int)d.D; a.R = (int)d.R; a.block = p.block; a.eps = d.eps;
    a.kx = kind_of(fx); a.kg = kind_of(fd); a.kw = norm ? kind_of(fw) : 0; a.ky = kind_of(fdx); a.kdw = want ? kind_of(fdw) : 0;
    a.fx = elem_fmt(fx); a.fg = elem_fmt(fd); a.fw = elem_fmt(norm ? fw : fx); a.fy = elem_fmt(fdx); a.fdw = elem_fmt(want ? fdw : fx);
    a.part = want ? (float*)workspace : nullptr;
    hipStream_t st = (hipStream_t)stream;
    PNN_DISPATCH_KIND(a.kx, (launch_heads<true, K>(st, p, d.neighbours != 0, a)))
    if (want) hipLaunchKernelGGL(heads_join_kernel, dim3((unsigned)((2 * d.D + 7) / 8)), dim3(256), 0, st, a, (int)p.groups);
    return hip_status(hipGetLastError());
}
