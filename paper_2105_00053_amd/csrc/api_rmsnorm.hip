// posit_rmsnorm_fwd / posit_rmsnorm_bwd / posit_scale_rows: the RMS norm of a residual stream, its gradient, and rows times scales.
#include "lm_codec.h"

namespace pnn {

struct NormFwd {
    const void *x, *res, *w;
    void *res_out, *y;
    float *scale, *rstd;
    int64_t cols, ldx, ldr, ldo, ldy;
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

// One row to a workgroup: the sum of squares, then the outputs from the stream read again.
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
    bool bad = false;
    if (a.scale) {
        top = block_max_u32(top, partu);
        bad = top >= 0x7F800000u;
        const int e = top == 0 ? 2 : ((top >> 23) ? (int)(top >> 23) - 127 : -118 - clz32(top));
        up = ldexpf(1.f, 2 - e);
        if (t == 0) a.scale[r] = bad ? f32_of_bits(0x7FC00000u) : ldexpf(rstd, e - 2);
    }
    for (int64_t j = t; j < a.cols; j += 256) {
        const float v = load_value(h, hrow + j, kh, fh) * load_value(a.w, j, a.kw, a.fw);
        store_value(a.y, r * a.ldy + j, a.ky, a.fy, bad ? f32_of_bits(0x7FC00000u) : v * up);
    }
}

struct NormBwd {
    const void *dy, *h, *w, *dres;
    const float* rstd;
    void *dx, *dw;
    int64_t rows, cols, lddy, ldh, lddr, lddx;
    int kd, kh, kw, kr, kx, kdw;
    ElemFmt fd, fh, fw, fr, fx, fdw;
};

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

__global__ __launch_bounds__(256) void scale_rows_kernel(const void* x, int64_t ldx, int kx, ElemFmt fx, const float* scale, void* y, int64_t ldy, int ky, ElemFmt fy,
                                                         int64_t cols) {
    const int64_t r = blockIdx.x;
    const float s = scale[r];
    for (int64_t j = threadIdx.x; j < cols; j += 256) store_value(y, r * ldy + j, ky, fy, s * load_value(x, r * ldx + j, kx, fx));
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
    NormFwd a = {x, res, w, res_out, y, scale, rstd, cols, ldx, ldr, ldo, ldy, eps, kind_of(fx), res ? kind_of(fres) : 0, kind_of(fw), kind_of(fy),
                 elem_fmt(fx), elem_fmt(res ? fres : fx), elem_fmt(fw), elem_fmt(fy)};
    hipLaunchKernelGGL(rmsnorm_fwd_kernel, dim3((unsigned)rows), dim3(256), 0, (hipStream_t)stream, a);
    return hip_status(hipGetLastError());
}

extern "C" size_t posit_rmsnorm_bwd_workspace(int64_t rows, int64_t cols) { return 0; }

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
    NormBwd a = {dy, h, w, dres, rstd, dx, dw, rows, cols, lddy, ldh, lddr, lddx, kind_of(fd), kind_of(fh), kind_of(fw), kind_of(dres ? fdres : fd), kind_of(fdx),
                 kind_of(dw ? fdw : fd), elem_fmt(fd), elem_fmt(fh), elem_fmt(fw), elem_fmt(dres ? fdres : fd), elem_fmt(fdx), elem_fmt(dw ? fdw : fd)};
    hipLaunchKernelGGL(rmsnorm_bwd_kernel, dim3((unsigned)rows), dim3(256), 0, (hipStream_t)stream, a);
    if (dw) hipLaunchKernelGGL(rmsnorm_dw_kernel, dim3((unsigned)((cols + 255) / 256)), dim3(256), 0, (hipStream_t)stream, a);
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
    hipLaunchKernelGGL(scale_rows_kernel, dim3((unsigned)rows), dim3(256), 0, (hipStream_t)stream, x, ldx, kind_of(fin), elem_fmt(fin), scale, y, ldy, kind_of(fout),
                       elem_fmt(fout), cols);
    return hip_status(hipGetLastError());
}
