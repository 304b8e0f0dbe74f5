// posit_rmsnorm_fwd / posit_rmsnorm_bwd / posit_scale_rows: the RMS norm of a residual stream, its gradient, and rows times scales.
//
// y = h w / sqrt(mean h^2 + eps), h = x + r.  Where rows are many the forward kernel is bound by the vector unit (decoding and rounding posits: busy 87 % of the
// cycles), the backward one by memory (vector unit 56 %); where they are few, by the launch.  16384 rows of 4096, 8-bit posits on a stream of 16-bit ones to
// bfloat16: forward 115 us in a row of calls (120 to 141 traced alone) for 470 MB, 4.1 TB/s where a large copy reaches 5.2; backward 110 to 114 for 537 MB, 4.9 TB/s.
// 4099 rows of 5119, odd pitches, bfloat16 stream to 8-bit posits with scales: 46 (traced 52; waves wait 62 % of their time for loads and stores of odd rows, even ones of 5120
// take 40); four rows of 2048: 5.
#include "lm_codec.h"

namespace pnn {

// The power of two that brings a row's largest magnitude (its binary32 word) into [4, 8), as two factors, since it is up to 2^151 where that magnitude is
// a subnormal number (`more` is 1 unless it is below 2^-125), and `rstd` times its inverse.  NaN for the first and the last where the row holds a NaN or an
// infinity.
__device__ __forceinline__ void norm_scale(uint32_t top, float rstd, float& up, float& more, float& scale) {
    const float nan = f32_of_bits(0x7FC00000u);
    const bool bad = top >= 0x7F800000u;
    const int e = top == 0 ? 2 : ((top >> 23) ? (int)(top >> 23) - 127 : -118 - clz32(top)), k = e < -125 ? 127 : 2 - e;
    up = bad ? nan : ldexpf(1.f, k);
    more = ldexpf(1.f, 2 - e - k);
    scale = bad ? nan : ldexpf(rstd, e - 2);
}

struct NormFwd {
    const void *x, *res, *w;
    void *res_out, *y;
    float *scale, *rstd;
    int64_t rows, cols, ldx, ldr, ldo, ldy;
    int64_t row0;  // of a launch with a row to a workgroup
    float eps;
    int kx, kr, kw, ky;
    ElemFmt fx, fr, fw, fy;
};

__device__ __forceinline__ float block_sum(float v, float* part) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return part[0] + part[1] + part[2] + part[3];
}

__device__ __forceinline__ uint32_t block_max_u32(uint32_t v, uint32_t* part) {
    v = wave_max_u32(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t m = part[0];
    for (int i = 1; i < 4; ++i) m = part[i] > m ? part[i] : m;
    return m;
}

// Values of 8-bit posits by look-up: 16 copies of each in LDS, so that the lanes of a wave meet few conflicts.  Pays where a workgroup
// has rows enough (a look-up takes 3 vector instructions, decoding 17; building the table as long as two rows).
constexpr int NORM_COPIES = 16, NORM_TABLE_ROWS = 4;
__device__ __forceinline__ void norm_table(uint32_t* table, ElemFmt f) {
    for (int e = threadIdx.x; e < 256 * NORM_COPIES / 4; e += blockDim.x) {
        const uint32_t v = bits_of_f32(posit_value(e / (NORM_COPIES / 4), f));
        ((uint4*)table)[e] = make_uint4(v, v, v, v);
    }
    __syncthreads();
}
template <int K>
__device__ __forceinline__ void norm_values(float (&v)[8], const Raw8& r, ElemFmt f, const uint32_t* table) {
    if (K == KIND_POSIT_U8 && table) {
        const uint32_t* mine = table + (threadIdx.x & (NORM_COPIES - 1));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = f32_of_bits(mine[((r.w[e / 4] >> (8 * (e & 3))) & 0xFFu) * NORM_COPIES]);
    } else {
        values8(v, r, K, f);
    }
}

// Sum (and maximum) over the T threads of a row; `slot` alternates, so that one barrier is enough.
__device__ __forceinline__ void norm_reduce(int T, float* part, uint32_t* partu, int slot, float& s, uint32_t& top, bool maximum) {
    s = wave_sum(s);
    if (maximum) top = wave_max_u32(top);
    if (T == 64) return;
    const int t = threadIdx.x, waves = T / 64, first = t / T * waves;
    if ((t & 63) == 0) {
        part[slot * 16 + (t >> 6)] = s;
        if (maximum) partu[slot * 16 + (t >> 6)] = top;
    }
    __syncthreads();
    s = 0.f;
    for (int i = 0; i < waves; ++i) s += part[slot * 16 + first + i];
    if (maximum) {
        top = 0;
        for (int i = 0; i < waves; ++i) top = partu[slot * 16 + first + i] > top ? partu[slot * 16 + first + i] : top;
    }
}

// Rows of up to 8192 elements, 8 to a thread: read once, with the next row's loads in flight, written once.  T threads (whole
// waves) to a row; the weights are decoded once for all rows of a workgroup.  KR < 0: no residual.
template <int KX, int KR>
__global__ __launch_bounds__(1024) void rmsnorm_fwd_rows_kernel(NormFwd a, int T) {
    __shared__ float part[32];
    __shared__ uint32_t partu[32];
    __shared__ uint32_t table_of[KX == KIND_POSIT_U8 ? 256 * NORM_COPIES : 1];
    const int t = threadIdx.x, group = t / T, j = (t - group * T) * 8, groups = blockDim.x / T, cols = (int)a.cols;
    const bool scaled = a.scale != nullptr;
    Raw8 x, res;
    auto load = [&](int64_t r) {
        const int left = r < a.rows ? cols - j : 0;
        load8(x, a.x, r * a.ldx + j, KX, left);
        if (KR >= 0) load8(res, a.res, r * a.ldr + j, KR, left);
    };
    const int64_t step = (int64_t)gridDim.x * groups;
    int64_t r = (int64_t)blockIdx.x * groups + group;
    load(r);
    float w[8];
    {
        Raw8 raw;
        load8(raw, a.w, j, a.kw, cols - j);
        values8(w, raw, a.kw, a.fw);
    }
    const uint32_t* table = nullptr;
    if (KX == KIND_POSIT_U8 && a.rows >= NORM_TABLE_ROWS * step) {
        norm_table(table_of, a.fx);
        table = table_of;
    }
    const float inv = 1.f / (float)cols;
    int slot = 0;
    // a workgroup's rows end together, so that its threads meet at the barriers
    for (int64_t r0 = (int64_t)blockIdx.x * groups; r0 < a.rows; r0 += step, r += step, slot ^= 1) {
        float h[8];
        norm_values<KX>(h, x, a.fx, table);
        if (KR >= 0) {
            float v[8];
            values8(v, res, KR, a.fr);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] += v[e];
            load(r + step);
            Raw8 out;
            raw8<true>(out, h, KR, a.fr);
            if (r < a.rows) store8(a.res_out, r * a.ldo + j, out, KR, cols - j);
        } else {
            load(r + step);
        }
        uint32_t top = 0;
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            ss = fmaf(h[e], h[e], ss);
            h[e] *= w[e];
        }
        if (scaled) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t m = bits_of_f32(h[e]) & 0x7FFFFFFFu;
                top = m > top ? m : top;
            }
        }
        norm_reduce(T, part, partu, slot, ss, top, scaled);
        if (r >= a.rows) continue;
        const float rstd = 1.f / sqrtf(ss * inv + a.eps);
        float up = rstd;
        if (scaled) {
            float more, scale;
            norm_scale(top, rstd, up, more, scale);
            if (j == 0) a.scale[r] = scale;
            if (more != 1.f) {
#pragma unroll
                for (int e = 0; e < 8; ++e) h[e] *= more;
            }
        }
        if (a.rstd && j == 0) a.rstd[r] = rstd;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] *= up;
        Raw8 out;
        raw8<false>(out, h, a.ky, a.fy);
        store8(a.y, r * a.ldy + j, out, a.ky, cols - j);
    }
}

// Longer rows, one to a workgroup: the sum of squares, then the outputs from the stream read again.  Element by element, kinds looked up for each: simple
// rather than fast.  4096 rows of 12288, 8-bit posits on a stream of 16-bit ones: 456 us for 352 MB; rmsnorm_bwd_kernel 426, rmsnorm_dw_kernel 2.7 ms (48 workgroups).
__global__ __launch_bounds__(256) void rmsnorm_fwd_kernel(NormFwd a) {
    __shared__ float part[4];
    __shared__ uint32_t partu[4];
    const int64_t r = a.row0 + blockIdx.x;
    const int t = threadIdx.x;
    const void* h = a.res ? a.res_out : a.x;
    const int kh = a.res ? a.kr : a.kx;
    const ElemFmt fh = a.res ? a.fr : a.fx;
    const int64_t hrow = r * (a.res ? a.ldo : a.ldx);
    float ss = 0.f;
    uint32_t top = 0;
    for (int64_t j = t; j < a.cols; j += 256) {
        float v = load_value(a.x, r * a.ldx + j, a.kx, a.fx);
        if (a.res) {
            store_value(a.res_out, hrow + j, a.kr, a.fr, v + load_value(a.res, r * a.ldr + j, a.kr, a.fr));
            v = load_value(a.res_out, hrow + j, a.kr, a.fr);
        }
        ss = fmaf(v, v, ss);
        const uint32_t m = bits_of_f32(v * load_value(a.w, j, a.kw, a.fw)) & 0x7FFFFFFFu;
        top = m > top ? m : top;
    }
    const float rstd = 1.f / sqrtf(block_sum(ss, part) / (float)a.cols + a.eps);
    if (a.rstd && t == 0) a.rstd[r] = rstd;
    float up = rstd, more = 1.f;
    if (a.scale) {
        top = block_max_u32(top, partu);
        float scale;
        norm_scale(top, rstd, up, more, scale);
        if (t == 0) a.scale[r] = scale;
    }
    for (int64_t j = t; j < a.cols; j += 256) {
        const float v = load_value(h, hrow + j, kh, fh) * load_value(a.w, j, a.kw, a.fw);
        store_value(a.y, r * a.ldy + j, a.ky, a.fy, v * more * up);
    }
}

struct NormBwd {
    const void *dy, *h, *w, *dres;
    const float* rstd;
    void *dx, *dw;
    int64_t rows, cols, lddy, ldh, lddr, lddx;
    int64_t row0;  // of a launch with a row to a workgroup
    int kd, kh, kw, kr, kx, kdw;
    ElemFmt fd, fh, fw, fr, fx, fdw;
    float* part;
};

// As the forward kernel for rows; each thread also sums its columns of dw over the workgroup's rows, and leaves the sums for
// rmsnorm_dw_join_kernel (one row of `part` to a workgroup, whose rows in parallel are joined in LDS).  KR < 0: no gradient past the norm; KR other than
// KD: its kind is a.kr.
template <int KD, int KH, int KR>
__global__ __launch_bounds__(1024) void rmsnorm_bwd_rows_kernel(NormBwd a, int T) {
    __shared__ float part[32];
    __shared__ float join[3 * 512];
    __shared__ uint32_t table_of[KD == KIND_POSIT_U8 ? 256 * NORM_COPIES : 1];
    const int t = threadIdx.x, group = t / T, tr = t - group * T, j = tr * 8, groups = blockDim.x / T, cols = (int)a.cols;
    const int kr = KR == KD ? KD : a.kr;
    Raw8 dy, hr, dres;
    float rs = 0.f;
    auto load = [&](int64_t r) {
        const int left = r < a.rows ? cols - j : 0;
        load8(dy, a.dy, r * a.lddy + j, KD, left);
        load8(hr, a.h, r * a.ldh + j, KH, left);
        if (KR >= 0) load8(dres, a.dres, r * a.lddr + j, kr, left);
        rs = r < a.rows ? a.rstd[r] : 0.f;
    };
    const int64_t step = (int64_t)gridDim.x * groups;
    int64_t r = (int64_t)blockIdx.x * groups + group;
    load(r);
    float w[8], dw[8];
    {
        Raw8 raw;
        load8(raw, a.w, j, a.kw, cols - j);
        values8(w, raw, a.kw, a.fw);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[e] = 0.f;
    const uint32_t* table = nullptr;
    if (KD == KIND_POSIT_U8 && a.rows >= NORM_TABLE_ROWS * step) {
        norm_table(table_of, a.fd);
        table = table_of;
    }
    const float inv = 1.f / (float)cols;
    int slot = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * groups; r0 < a.rows; r0 += step, r += step, slot ^= 1) {
        float g[8], h[8], past[8];
        const float rstd = rs;
        const bool live = r < a.rows;
        norm_values<KD>(g, dy, a.fd, table);
        values8(h, hr, KH, a.fh);
        if (KR >= 0) values8(past, dres, kr, a.fr);
        load(r + step);
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            dw[e] = live ? fmaf(g[e] * rstd, h[e], dw[e]) : dw[e];
            g[e] *= w[e];
            s = fmaf(g[e], h[e], s);
        }
        uint32_t none = 0;
        norm_reduce(T, part, nullptr, slot, s, none, false);
        if (!live) continue;
        const float k = s * inv * rstd * rstd * rstd;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = rstd * g[e] - k * h[e];
            if (KR >= 0) v[e] += past[e];
        }
        Raw8 out;
        raw8<false>(out, v, a.kx, a.fx);
        store8(a.dx, r * a.lddx + j, out, a.kx, cols - j);
    }
    if (!a.dw) return;
    // groups of threads only where a workgroup is 256 threads: 4 of 64 or 2 of 128
    if (groups > 1) {
        if (group > 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) join[((group - 1) * 8 + e) * T + tr] = dw[e];
        }
        __syncthreads();
        if (group > 0) return;
        for (int x = 0; x < groups - 1; ++x)
#pragma unroll
            for (int e = 0; e < 8; ++e) dw[e] += join[(x * 8 + e) * T + tr];
    }
    float* const out = a.part + (int64_t)blockIdx.x * a.cols + j;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (j + e < cols) out[e] = dw[e];
}

// Columns of the partial sums: 32 columns to a workgroup, 32 threads to a column, in a fixed order.
__global__ __launch_bounds__(1024) void rmsnorm_dw_join_kernel(const float* part, int groups, int64_t cols, void* dw, int kind, ElemFmt f) {
    __shared__ float sums[32][33];
    const int c = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t j = (int64_t)blockIdx.x * 32 + c;
    float s = 0.f;
    if (j < cols) {
        int g = y;
        for (; g + 96 < groups; g += 128) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = part[(int64_t)(g + 32 * i) * cols + j];
            s += (v[0] + v[1]) + (v[2] + v[3]);
        }
        for (; g < groups; g += 32) s += part[(int64_t)g * cols + j];
    }
    sums[y][c] = s;
    __syncthreads();
    if (y == 0 && j < cols) {
        for (int k = 1; k < 32; ++k) s += sums[k][c];
        store_value(dw, j, kind, f, s);
    }
}

// Longer rows.
__global__ __launch_bounds__(256) void rmsnorm_bwd_kernel(NormBwd a) {
    __shared__ float part[4];
    const int64_t r = a.row0 + blockIdx.x;
    const int t = threadIdx.x;
    float s = 0.f;
    for (int64_t j = t; j < a.cols; j += 256)
        s = fmaf(load_value(a.dy, r * a.lddy + j, a.kd, a.fd) * load_value(a.w, j, a.kw, a.fw), load_value(a.h, r * a.ldh + j, a.kh, a.fh), s);
    const float rs = a.rstd[r];
    const float c = block_sum(s, part) / (float)a.cols * rs * rs * rs;
    for (int64_t j = t; j < a.cols; j += 256) {
        const float g = load_value(a.dy, r * a.lddy + j, a.kd, a.fd) * load_value(a.w, j, a.kw, a.fw);
        float v = rs * g - c * load_value(a.h, r * a.ldh + j, a.kh, a.fh);
        if (a.dres) v += load_value(a.dres, r * a.lddr + j, a.kr, a.fr);
        store_value(a.dx, r * a.lddx + j, a.kx, a.fx, v);
    }
}

__global__ __launch_bounds__(256) void rmsnorm_dw_kernel(NormBwd a) {
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= a.cols) return;
    float s = 0.f;
    for (int64_t r = 0; r < a.rows; ++r)
        s = fmaf(load_value(a.dy, r * a.lddy + j, a.kd, a.fd) * a.rstd[r], load_value(a.h, r * a.ldh + j, a.kh, a.fh), s);
    store_value(a.dw, j, a.kdw, a.fdw, s);
}

// 8 elements to a thread; 4099 x 5119 in 8-bit posits to binary32 21 us, 5 TB/s (both sides unaligned), four rows of 2048 2.
__global__ __launch_bounds__(256) void scale_rows_kernel(const void* x, int64_t ldx, int kx, ElemFmt fx, const float* scale, void* y, int64_t ldy, int ky, ElemFmt fy,
                                                         int64_t rows, int64_t cols, uint32_t vectors) {
    const uint32_t id = blockIdx.x * 256u + threadIdx.x, r = id / vectors;
    const int64_t j = (int64_t)(id - r * vectors) * 8;
    if (r >= rows) return;
    const int left = cols - j < 8 ? (int)(cols - j) : 8;
    Raw8 raw;
    load8(raw, x, r * ldx + j, kx, left);
    const float s = scale[r];
    float v[8];
    values8(v, raw, kx, fx);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= s;
    raw8<false>(raw, v, ky, fy);
    store8(y, r * ldy + j, raw, ky, left);
}

// Threads to a row (whole waves of them), threads and number of workgroups.  Rows beyond 8 elements a thread of the largest workgroup have kernels
// of their own.
struct NormPlan {
    bool rows;
    int T, threads;
    unsigned groups;
};
inline NormPlan norm_plan(int64_t rows, int64_t cols, int waves) {
    NormPlan p = {cols <= 8192, 1024, 1024, 0};
    if (p.rows) p.T = (int)((cols + 511) / 512) * 64;
    p.threads = p.T == 64 || p.T == 128 ? 256 : p.T;
    // as many workgroups as the chip holds, each walking over rows; `waves` of them to a compute unit, by the kernels' registers
    const int64_t want = (rows + p.threads / p.T - 1) / (p.threads / p.T), most = 256 * (waves * 64 / p.threads);
    p.groups = (unsigned)(want < most ? want : most);
    return p;
}

// What the kernels' registers leave room for (forward up to 72 of 512, backward up to 128).  us in a row of calls with 32, 28 and 16 waves to a compute unit: forward,
// bfloat16 stream to 8-bit posits with scales, 4099 rows of 5119, 52, 46 and 67; 16384 of 4096, 101, 98 and 108; 16-bit posit stream to bfloat16, 60, 55 and 76; 116, 115 and 121;
// backward (with dw) of the latter, 74, 69 and 63; 93, 90 and 87; 2000 rows of 3000, 31, 27 and 22.
constexpr int NORM_FWD_WAVES = 28, NORM_BWD_WAVES = 16;

template <int KX>
void launch_fwd_rows(hipStream_t st, const NormPlan& p, const NormFwd& a) {
    const dim3 g(p.groups), b(p.threads);
    if (!a.res) {
        hipLaunchKernelGGL((rmsnorm_fwd_rows_kernel<KX, -1>), g, b, 0, st, a, p.T);
        return;
    }
    PNN_DISPATCH_KIND(a.kr, hipLaunchKernelGGL((rmsnorm_fwd_rows_kernel<KX, K>), g, b, 0, st, a, p.T))
}

template <int KD, int KH>
void launch_bwd_rows(hipStream_t st, const NormPlan& p, const NormBwd& a) {
    const dim3 g(p.groups), b(p.threads);
    constexpr int OTHER = KD == KIND_F32 ? KIND_BF16 : KIND_F32;  // any kind that is not KD
    if (!a.dres) hipLaunchKernelGGL((rmsnorm_bwd_rows_kernel<KD, KH, -1>), g, b, 0, st, a, p.T);
    else if (a.kr == KD) hipLaunchKernelGGL((rmsnorm_bwd_rows_kernel<KD, KH, KD>), g, b, 0, st, a, p.T);
    else hipLaunchKernelGGL((rmsnorm_bwd_rows_kernel<KD, KH, OTHER>), g, b, 0, st, a, p.T);
}
template <int KD>
void launch_bwd_rows_of(hipStream_t st, const NormPlan& p, const NormBwd& a) {
    PNN_DISPATCH_KIND(a.kh, (launch_bwd_rows<KD, K>(st, p, a)))
}

}  // namespace pnn

using namespace pnn;

extern "C" int posit_rmsnorm_fwd(void* stream, int fx, int fres, int fw, int fy, int64_t rows, int64_t cols, const void* x, int64_t ldx, const void* res,
                                 int64_t ldr, const void* w, float eps, void* res_out, int64_t ldo, void* y, int64_t ldy, float* scale, float* rstd) {
    if (rows < 0 || cols < 0 || !(eps >= 0.f) || ldx < cols || ldy < cols || (res && (ldr < cols || ldo < cols))) return PNN_EINVAL;
    for (int f : {fx, fw, fy, res ? fres : fx})
        if (const int s = element_status(f)) return s;
    if (rows == 0 || cols == 0) return PNN_OK;
    if (!x || !w || !y || (res && !res_out)) return PNN_EINVAL;
    if (rows >= ((int64_t)1 << 31) || cols >= ((int64_t)1 << 31)) return PNN_EUNSUPPORTED;
    discard_stale_hip_error();
    NormFwd a = {x, res, w, res_out, y, scale, rstd, rows, cols, ldx, ldr, ldo, ldy, 0, eps, kind_of(fx), res ? kind_of(fres) : 0, kind_of(fw), kind_of(fy),
                 elem_fmt(fx), elem_fmt(res ? fres : fx), elem_fmt(fw), elem_fmt(fy)};
    hipStream_t st = (hipStream_t)stream;
    const NormPlan p = norm_plan(rows, cols, NORM_FWD_WAVES);
    if (p.rows) {
        PNN_DISPATCH_KIND(a.kx, launch_fwd_rows<K>(st, p, a))
    } else {
        for (const int64_t most = most_workgroups(256); a.row0 < rows; a.row0 += most)
            hipLaunchKernelGGL(rmsnorm_fwd_kernel, dim3((unsigned)(rows - a.row0 < most ? rows - a.row0 : most)), dim3(256), 0, st, a);
    }
    return hip_status(hipGetLastError());
}

extern "C" size_t posit_rmsnorm_bwd_workspace(int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0 || cols > 8192) return 0;
    return (size_t)norm_plan(rows, cols, NORM_BWD_WAVES).groups * (size_t)cols * 4;
}

extern "C" int posit_rmsnorm_bwd(void* stream, int fd, int fh, int fw, int fdres, int fdx, int fdw, int64_t rows, int64_t cols, const void* dy, int64_t lddy,
                                 const void* h, int64_t ldh, const void* w, const float* rstd, const void* dres, int64_t lddr, void* dx, int64_t lddx, void* dw,
                                 void* workspace, size_t workspace_bytes) {
    if (rows < 0 || cols < 0 || lddy < cols || ldh < cols || lddx < cols || (dres && lddr < cols)) return PNN_EINVAL;
    for (int f : {fd, fh, fw, fdx, dres ? fdres : fd, dw ? fdw : fd})
        if (const int s = element_status(f)) return s;
    if (rows == 0 || cols == 0) return PNN_OK;
    if (!dy || !h || !w || !rstd || !dx) return PNN_EINVAL;
    if (rows >= ((int64_t)1 << 31) || cols >= ((int64_t)1 << 31)) return PNN_EUNSUPPORTED;
    discard_stale_hip_error();
    const size_t need = dw ? posit_rmsnorm_bwd_workspace(rows, cols) : 0;
    if (need > 0 && (!workspace || workspace_bytes < need)) return PNN_EWORKSPACE;
    if (need > 0 && !aligned(workspace, 16)) return PNN_EINVAL;
    NormBwd a = {dy, h, w, dres, rstd, dx, dw, rows, cols, lddy, ldh, lddr, lddx, 0, kind_of(fd), kind_of(fh), kind_of(fw), kind_of(dres ? fdres : fd), kind_of(fdx),
                 kind_of(dw ? fdw : fd), elem_fmt(fd), elem_fmt(fh), elem_fmt(fw), elem_fmt(dres ? fdres : fd), elem_fmt(fdx), elem_fmt(dw ? fdw : fd), (float*)workspace};
    hipStream_t st = (hipStream_t)stream;
    const NormPlan p = norm_plan(rows, cols, NORM_BWD_WAVES);
    if (p.rows) {
        PNN_DISPATCH_KIND(a.kd, launch_bwd_rows_of<K>(st, p, a))
        if (dw) hipLaunchKernelGGL(rmsnorm_dw_join_kernel, dim3((unsigned)((cols + 31) / 32)), dim3(1024), 0, st, a.part, (int)p.groups, cols, dw, a.kdw, a.fdw);
    } else {
        for (const int64_t most = most_workgroups(256); a.row0 < rows; a.row0 += most)
            hipLaunchKernelGGL(rmsnorm_bwd_kernel, dim3((unsigned)(rows - a.row0 < most ? rows - a.row0 : most)), dim3(256), 0, st, a);
        if (dw) hipLaunchKernelGGL(rmsnorm_dw_kernel, dim3((unsigned)((cols + 255) / 256)), dim3(256), 0, st, a);
    }
    return hip_status(hipGetLastError());
}

extern "C" int posit_scale_rows(void* stream, int fin, int fout, int64_t rows, int64_t cols, const void* x, int64_t ldx, const float* scale, void* y, int64_t ldy) {
    if (rows < 0 || cols < 0 || ldx < cols || ldy < cols) return PNN_EINVAL;
    for (int f : {fin, fout})
        if (const int s = element_status(f)) return s;
    if (rows == 0 || cols == 0) return PNN_OK;
    if (!x || !scale || !y) return PNN_EINVAL;
    if (rows >= ((int64_t)1 << 31)) return PNN_EUNSUPPORTED;
    discard_stale_hip_error();
    // threads are numbered in 32 bits: rows in as many launches as that takes
    const int64_t vectors = (cols + 7) / 8, most = (((int64_t)1 << 31) - 256) / vectors;
    if (most == 0) return PNN_EUNSUPPORTED;
    for (int64_t r = 0; r < rows; r += most) {
        const int64_t n = rows - r < most ? rows - r : most;
        hipLaunchKernelGGL(scale_rows_kernel, dim3((unsigned)((n * vectors + 255) / 256)), dim3(256), 0, (hipStream_t)stream, (const char*)x + r * ldx * element_bytes(fin), ldx,
                           kind_of(fin), elem_fmt(fin), scale + r, (char*)y + r * ldy * element_bytes(fout), ldy, kind_of(fout), elem_fmt(fout), n, cols, (uint32_t)vectors);
    }
    return hip_status(hipGetLastError());
}
