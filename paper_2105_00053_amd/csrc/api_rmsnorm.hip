// posit_rmsnorm_fwd / posit_rmsnorm_bwd / posit_scale_rows: the RMS norm of a residual stream, its gradient, and rows times scales.
#include "lm_codec.h"

namespace pnn {

// The power of two that brings a row's largest magnitude (its binary32 word) into [4, 8), and the one that undoes it.  True, with NaN
// for the first, where the row holds a NaN or an infinity.
__device__ __forceinline__ bool norm_scale(uint32_t top, float& up, float& down) {
    const bool bad = top >= 0x7F800000u;
    const int e = top == 0 ? 2 : ((top >> 23) ? (int)(top >> 23) - 127 : -118 - clz32(top));
    up = bad ? f32_of_bits(0x7FC00000u) : ldexpf(1.f, 2 - e);
    down = ldexpf(1.f, e - 2);
    return bad;
}

struct NormFwd {
    const void *x, *res, *w;
    void *res_out, *y;
    float *scale, *rstd;
    int64_t rows, cols, ldx, ldr, ldo, ldy;
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

// Rows that fit the registers of T threads, 8 C elements to a thread: read once, with the next row's loads in flight, written once.
// The weights are decoded once for all rows of a workgroup.
template <int T, int C>
__global__ __launch_bounds__(256) void rmsnorm_fwd_rows_kernel(NormFwd a) {
    __shared__ float part[2][4];
    __shared__ uint32_t partu[2][4];
    const int t = threadIdx.x, tr = t % T, cols = (int)a.cols;
    const bool add = a.res != nullptr;
    float w[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        Raw8 r;
        load8(r, a.w, (c * T + tr) * 8, a.kw, cols - (c * T + tr) * 8);
        values8(w[c], r, a.kw, a.fw);
    }
    const float inv = 1.f / (float)cols;
    Raw8 x[C], res[C];
    auto load = [&](int64_t r) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int j = (c * T + tr) * 8, left = r < a.rows ? cols - j : 0;
            load8(x[c], a.x, r * a.ldx + j, a.kx, left);
            if (add) load8(res[c], a.res, r * a.ldr + j, a.kr, left);
        }
    };
    const int64_t step = (int64_t)gridDim.x * (256 / T);
    int64_t r = (int64_t)blockIdx.x * (256 / T) + t / T;
    load(r);
    // a workgroup's rows end together, so that its threads meet at the barriers
    for (int64_t r0 = (int64_t)blockIdx.x * (256 / T), n = 0; r0 < a.rows; r0 += step, r += step, ++n) {
        float h[C][8];
        float ss = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            values8(h[c], x[c], a.kx, a.fx);
            if (add) {
                float v[8];
                values8(v, res[c], a.kr, a.fr);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[c][e] += v[e];
                const int j = (c * T + tr) * 8;
                Raw8 out;
                raw8<true>(out, h[c], a.kr, a.fr);
                if (r < a.rows) store8(a.res_out, r * a.ldo + j, out, a.kr, cols - j);
            }
        }
        load(r + step);
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ss = fmaf(h[c][e], h[c][e], ss);
                h[c][e] *= w[c][e];
                if (a.scale) {
                    const uint32_t m = bits_of_f32(h[c][e]) & 0x7FFFFFFFu;
                    top = m > top ? m : top;
                }
            }
        ss = wave_sum(ss);
        if (a.scale) top = wave_max_u32(top);
        if (T > 64) {
            if ((t & 63) == 0) {
                part[n & 1][t >> 6] = ss;
                partu[n & 1][t >> 6] = top;
            }
            __syncthreads();
            const float* p = part[n & 1];
            const uint32_t* u = partu[n & 1];
            ss = (p[0] + p[1]) + (p[2] + p[3]);
            const uint32_t u0 = u[0] > u[1] ? u[0] : u[1], u1 = u[2] > u[3] ? u[2] : u[3];
            top = u0 > u1 ? u0 : u1;
        }
        if (r >= a.rows) continue;
        const float rstd = 1.f / sqrtf(ss * inv + a.eps);
        float up = rstd;
        if (a.scale) {
            float down;
            const bool bad = norm_scale(top, up, down);
            if (tr == 0) a.scale[r] = bad ? f32_of_bits(0x7FC00000u) : rstd * down;
        }
        if (a.rstd && tr == 0) a.rstd[r] = rstd;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int j = (c * T + tr) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) h[c][e] *= up;
            Raw8 out;
            raw8<false>(out, h[c], a.ky, a.fy);
            store8(a.y, r * a.ldy + j, out, a.ky, cols - j);
        }
    }
}

// Longer rows, one to a workgroup: the sum of squares, then the outputs from the stream read again.
__global__ __launch_bounds__(256) void rmsnorm_fwd_kernel(NormFwd a) {
    __shared__ float part[4];
    __shared__ uint32_t partu[4];
    const int64_t r = blockIdx.x;
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
    float up = rstd;
    if (a.scale) {
        top = block_max_u32(top, partu);
        float down;
        const bool bad = norm_scale(top, up, down);
        if (t == 0) a.scale[r] = bad ? f32_of_bits(0x7FC00000u) : rstd * down;
    }
    for (int64_t j = t; j < a.cols; j += 256) {
        const float v = load_value(h, hrow + j, kh, fh) * load_value(a.w, j, a.kw, a.fw);
        store_value(a.y, r * a.ldy + j, a.ky, a.fy, v * up);
    }
}

struct NormBwd {
    const void *dy, *h, *w, *dres;
    const float* rstd;
    void *dx, *dw;
    int64_t rows, cols, lddy, ldh, lddr, lddx;
    int kd, kh, kw, kr, kx, kdw;
    ElemFmt fd, fh, fw, fr, fx, fdw;
    float* part;
};

// As the forward kernel for rows; each thread also sums its columns of dw over the workgroup's rows, and leaves the sums for
// rmsnorm_dw_join_kernel (one row of `part` to a workgroup; its waves are joined in LDS where a row is a wave's).
template <int T, int C>
__global__ __launch_bounds__(256) void rmsnorm_bwd_rows_kernel(NormBwd a) {
    __shared__ float sums[2][4];
    __shared__ float join[T == 64 ? 3 * C * 512 : 1];
    const int t = threadIdx.x, tr = t % T, cols = (int)a.cols;
    float w[C][8], dw[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        Raw8 r;
        load8(r, a.w, (c * T + tr) * 8, a.kw, cols - (c * T + tr) * 8);
        values8(w[c], r, a.kw, a.fw);
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[c][e] = 0.f;
    }
    const float inv = 1.f / (float)cols;
    Raw8 dy[C], hr[C], dres[C];
    float rs = 0.f;
    auto load = [&](int64_t r) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int j = (c * T + tr) * 8, left = r < a.rows ? cols - j : 0;
            load8(dy[c], a.dy, r * a.lddy + j, a.kd, left);
            load8(hr[c], a.h, r * a.ldh + j, a.kh, left);
            if (a.dres) load8(dres[c], a.dres, r * a.lddr + j, a.kr, left);
        }
        rs = r < a.rows ? a.rstd[r] : 0.f;
    };
    const int64_t step = (int64_t)gridDim.x * (256 / T);
    int64_t r = (int64_t)blockIdx.x * (256 / T) + t / T;
    load(r);
    for (int64_t r0 = (int64_t)blockIdx.x * (256 / T), n = 0; r0 < a.rows; r0 += step, r += step, ++n) {
        float g[C][8], h[C][8], past[C][8];
        float s = 0.f;
        const float rstd = rs;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            values8(g[c], dy[c], a.kd, a.fd);
            values8(h[c], hr[c], a.kh, a.fh);
#pragma unroll
            for (int e = 0; e < 8; ++e) past[c][e] = 0.f;
            if (a.dres) values8(past[c], dres[c], a.kr, a.fr);
        }
        load(r + step);
        const bool live = r < a.rows;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (live) dw[c][e] = fmaf(g[c][e] * rstd, h[c][e], dw[c][e]);
                g[c][e] *= w[c][e];
                s = fmaf(g[c][e], h[c][e], s);
            }
        s = wave_sum(s);
        if (T > 64) {
            if ((t & 63) == 0) sums[n & 1][t >> 6] = s;
            __syncthreads();
            const float* p = sums[n & 1];
            s = (p[0] + p[1]) + (p[2] + p[3]);
        }
        if (!live) continue;
        const float k = s * inv * rstd * rstd * rstd;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int j = (c * T + tr) * 8;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = rstd * g[c][e] - k * h[c][e] + past[c][e];
            Raw8 out;
            raw8<false>(out, v, a.kx, a.fx);
            store8(a.dx, r * a.lddx + j, out, a.kx, cols - j);
        }
    }
    if (!a.dw) return;
    if (T == 64) {
        const int wave = t >> 6;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (wave > 0) join[((wave - 1) * C * 8 + c * 8 + e) * 64 + tr] = dw[c][e];
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int x = 0; x < 3; ++x)
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) dw[c][e] += join[(x * C * 8 + c * 8 + e) * 64 + tr];
    }
    float* const out = a.part + (int64_t)blockIdx.x * a.cols;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if ((c * T + tr) * 8 + e < cols) out[(c * T + tr) * 8 + e] = dw[c][e];
}

// Columns of the partial sums: 16 columns to a workgroup, 16 threads to a column, in a fixed order.
__global__ __launch_bounds__(256) void rmsnorm_dw_join_kernel(const float* part, int64_t groups, int64_t cols, void* dw, int kind, ElemFmt f) {
    __shared__ float sums[16][17];
    const int c = threadIdx.x & 15, y = threadIdx.x >> 4;
    const int64_t j = (int64_t)blockIdx.x * 16 + c;
    float s = 0.f;
    if (j < cols)
        for (int64_t g = y; g < groups; g += 16) s += part[g * cols + j];
    sums[y][c] = s;
    __syncthreads();
    if (y == 0 && j < cols) {
        for (int k = 1; k < 16; ++k) s += sums[k][c];
        store_value(dw, j, kind, f, s);
    }
}

// Longer rows.
__global__ __launch_bounds__(256) void rmsnorm_bwd_kernel(NormBwd a) {
    __shared__ float part[4];
    const int64_t r = blockIdx.x;
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

// 8 elements to a thread
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

// Threads to a row and vectors of 8 to a thread, by the row's length: a wave as long as a row is 16 elements a thread, else a
// workgroup.  BEFORE runs where one of them applies, with the grid's size in `groups`.
#define PNN_NORM_LAUNCH(KERNEL, T, C, BEFORE)                                                         \
    {                                                                                                  \
        const int64_t want = (rows + 256 / T - 1) / (256 / T);                                          \
        const unsigned groups = (unsigned)(want < NORM_GROUPS ? want : NORM_GROUPS);                      \
        BEFORE;                                                                                          \
        hipLaunchKernelGGL((KERNEL<T, C>), dim3(groups), dim3(256), 0, st, a);                             \
    }
#define PNN_NORM_ROWS(cols, KERNEL, BEFORE)                          \
    if (cols <= 512) PNN_NORM_LAUNCH(KERNEL, 64, 1, BEFORE)           \
    else if (cols <= 1024) PNN_NORM_LAUNCH(KERNEL, 64, 2, BEFORE)      \
    else if (cols <= 2048) PNN_NORM_LAUNCH(KERNEL, 256, 1, BEFORE)      \
    else if (cols <= 4096) PNN_NORM_LAUNCH(KERNEL, 256, 2, BEFORE)       \
    else if (cols <= 8192) PNN_NORM_LAUNCH(KERNEL, 256, 4, BEFORE)
constexpr int64_t NORM_GROUPS = 1024;

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
    NormFwd a = {x, res, w, res_out, y, scale, rstd, rows, cols, ldx, ldr, ldo, ldy, eps, kind_of(fx), res ? kind_of(fres) : 0, kind_of(fw), kind_of(fy),
                 elem_fmt(fx), elem_fmt(res ? fres : fx), elem_fmt(fw), elem_fmt(fy)};
    hipStream_t st = (hipStream_t)stream;
    PNN_NORM_ROWS(cols, rmsnorm_fwd_rows_kernel, (void)0)
    else hipLaunchKernelGGL(rmsnorm_fwd_kernel, dim3((unsigned)rows), dim3(256), 0, st, a);
    return hip_status(hipGetLastError());
}

extern "C" size_t posit_rmsnorm_bwd_workspace(int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0 || cols > 8192) return 0;
    const int64_t per = cols <= 1024 ? 4 : 1, want = (rows + per - 1) / per;
    return (size_t)((want < NORM_GROUPS ? want : NORM_GROUPS) * cols * 4);
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
    NormBwd a = {dy, h, w, dres, rstd, dx, dw, rows, cols, lddy, ldh, lddr, lddx, kind_of(fd), kind_of(fh), kind_of(fw), kind_of(dres ? fdres : fd), kind_of(fdx),
                 kind_of(dw ? fdw : fd), elem_fmt(fd), elem_fmt(fh), elem_fmt(fw), elem_fmt(dres ? fdres : fd), elem_fmt(fdx), elem_fmt(dw ? fdw : fd), (float*)workspace};
    hipStream_t st = (hipStream_t)stream;
    unsigned used = 0;
    PNN_NORM_ROWS(cols, rmsnorm_bwd_rows_kernel, used = groups)
    else {
        hipLaunchKernelGGL(rmsnorm_bwd_kernel, dim3((unsigned)rows), dim3(256), 0, st, a);
        if (dw) hipLaunchKernelGGL(rmsnorm_dw_kernel, dim3((unsigned)((cols + 255) / 256)), dim3(256), 0, st, a);
    }
    if (dw && used) hipLaunchKernelGGL(rmsnorm_dw_join_kernel, dim3((unsigned)((cols + 15) / 16)), dim3(256), 0, st, a.part, (int64_t)used, cols, dw, a.kdw, a.fdw);
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
