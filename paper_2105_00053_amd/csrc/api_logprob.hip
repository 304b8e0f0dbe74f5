// posit_token_logprob_fwd / posit_token_logprob_bwd: log probabilities of given tokens, entropy, top alternatives, and the gradient.
#include "lm_codec.h"

namespace pnn {

struct LogprobFwd {
    const void* z;
    const int32_t* target;
    float *logprob, *lse, *entropy, *top_logprob;
    int32_t* top_index;
    int64_t vocab, ldz;
    float tau;
    int top, kind;
    ElemFmt f;
};

// Order of values as integers; -0 as +0.
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t b = bits_of_f32(v + 0.f);
    return b ^ (((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of_order(uint32_t o) { return f32_of_bits(o & 0x80000000u ? o ^ 0x80000000u : ~o); }

__device__ __forceinline__ float block4(float v, float* part, bool maximum) {
    v = maximum ? wave_max(v) : wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return maximum ? fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])) : part[0] + part[1] + part[2] + part[3];
}

// One row to a workgroup: maximum, sums, then one pass for each alternative.
__global__ __launch_bounds__(256) void logprob_fwd_kernel(LogprobFwd a) {
    __shared__ float part[4];
    __shared__ unsigned long long best[4];
    const int64_t r = blockIdx.x;
    const int t = threadIdx.x;
    const float inf = f32_of_bits(0x7F800000u), nan = f32_of_bits(0x7FC00000u);
    float m = -inf, bad = 0.f;
    for (int64_t j = t; j < a.vocab; j += 256) {
        const float z = load_value(a.z, r * a.ldz + j, a.kind, a.f) * a.tau;
        if (!(z < inf)) bad = 1.f;
        m = fmaxf(m, z);
    }
    m = block4(m, part, true);
    bad = block4(bad, part, true);
    const bool empty = m == -inf;
    float s = 0.f, u = 0.f;
    for (int64_t j = t; j < a.vocab; j += 256) {
        const float d = load_value(a.z, r * a.ldz + j, a.kind, a.f) * a.tau - m, e = expf(d);
        s += e;
        u += e > 0.f ? e * d : 0.f;
    }
    s = block4(s, part, false);
    u = block4(u, part, false);
    const float logs = logf(s);
    const float lse = bad > 0.f ? nan : (empty ? -inf : m + logs);
    if (t == 0) {
        if (a.lse) a.lse[r] = lse;
        if (a.entropy) a.entropy[r] = bad > 0.f ? nan : (empty ? 0.f : logs - u / s);
        if (a.logprob) {
            const int32_t y = a.target[r];
            float lp = 0.f;
            if (bad > 0.f || y >= a.vocab) lp = nan;
            else if (y >= 0) lp = empty ? -inf : (load_value(a.z, r * a.ldz + y, a.kind, a.f) * a.tau - m) - logs;
            if (y < 0 && !(bad > 0.f)) lp = 0.f;
            a.logprob[r] = lp;
        }
    }
    unsigned long long last = ~0ull;
    for (int k = 0; k < a.top; ++k) {
        unsigned long long b = 0;
        for (int64_t j = t; j < a.vocab; j += 256) {
            const float z = load_value(a.z, r * a.ldz + j, a.kind, a.f);
            const unsigned long long key = ((unsigned long long)order_of(z) << 32) | (uint32_t)~(uint32_t)j;
            if (z > -inf && key < last && key > b) b = key;
        }
        for (int q = 32; q >= 1; q >>= 1) {
            const unsigned long long o = __shfl_xor(b, q, 64);
            b = o > b ? o : b;
        }
        __syncthreads();
        if ((t & 63) == 0) best[t >> 6] = b;
        __syncthreads();
        for (int q = 0; q < 4; ++q) b = best[q] > b ? best[q] : b;
        if (t == 0) {
            const bool none = b == 0 || bad > 0.f;
            a.top_index[r * a.top + k] = none ? -1 : (int32_t)~(uint32_t)b;
            a.top_logprob[r * a.top + k] = bad > 0.f ? nan : (none ? -inf : (value_of_order((uint32_t)(b >> 32)) * a.tau - m) - logs);
        }
        last = b;
        if (b == 0) last = 0;
    }
}

struct LogprobBwd {
    const void* z;
    const int32_t* target;
    const float *lse, *entropy, *g_lp, *g_ent;
    void* dz;
    int64_t vocab, ldz, ldg;
    float tau;
    int kz, kg;
    ElemFmt fz, fg;
};

__global__ __launch_bounds__(256) void logprob_bwd_kernel(LogprobBwd a) {
    const int64_t r = blockIdx.x;
    const float lse = a.lse[r], inf = f32_of_bits(0x7F800000u);
    const float gl = a.g_lp ? a.g_lp[r] : 0.f, ge = a.g_ent ? a.g_ent[r] : 0.f, h = a.g_ent ? a.entropy[r] : 0.f;
    const int32_t y = a.g_lp ? a.target[r] : -1;
    const float g1 = y < 0 ? 0.f : (y >= a.vocab ? f32_of_bits(0x7FC00000u) : gl);
    for (int64_t j = threadIdx.x; j < a.vocab; j += 256) {
        const float lp = lse == -inf ? -inf : load_value(a.z, r * a.ldz + j, a.kz, a.fz) * a.tau - lse, p = expf(lp);
        float g = g1 * ((j == y ? 1.f : 0.f) - p);
        if (a.g_ent && !(p <= 0.f)) g -= ge * p * (lp + h);
        store_value(a.dz, r * a.ldg + j, a.kg, a.fg, a.tau * g);
    }
}

}  // namespace pnn

using namespace pnn;

extern "C" size_t posit_token_logprob_workspace(int fz, int64_t rows, int64_t vocab, int top) { return 0; }

extern "C" int posit_token_logprob_fwd(void* stream, int fz, int64_t rows, int64_t vocab, const void* logits, int64_t ldz, const int32_t* targets,
                                       float inv_temperature, int top, float* logprob, float* lse, float* entropy, float* top_logprob, int32_t* top_index,
                                       void* workspace, size_t workspace_bytes) {
    if (rows < 0 || vocab < 0 || ldz < vocab || top < 0 || !(inv_temperature > 0.f && inv_temperature <= 3.4028235e38f)) return PNN_EINVAL;
    if (const int s = element_status(fz)) return s;
    if (top > 64 || rows >= ((int64_t)1 << 31) || vocab >= ((int64_t)1 << 31)) return PNN_EUNSUPPORTED;
    if (rows == 0 || vocab == 0) return PNN_OK;
    if (!logits || (logprob && !targets) || (top > 0 && (!top_logprob || !top_index)) || (!logprob && !lse && !entropy && top == 0)) return PNN_EINVAL;
    discard_stale_hip_error();
    const LogprobFwd a = {logits, targets, logprob, lse, entropy, top_logprob, top_index, vocab, ldz, inv_temperature, top, kind_of(fz), elem_fmt(fz)};
    hipLaunchKernelGGL(logprob_fwd_kernel, dim3((unsigned)rows), dim3(256), 0, (hipStream_t)stream, a);
    return hip_status(hipGetLastError());
}

extern "C" int posit_token_logprob_bwd(void* stream, int fz, int fg, int64_t rows, int64_t vocab, const void* logits, int64_t ldz, const int32_t* targets,
                                       float inv_temperature, const float* lse, const float* entropy, const float* g_logprob, const float* g_entropy,
                                       void* dlogits, int64_t ldg) {
    if (rows < 0 || vocab < 0 || ldz < vocab || ldg < vocab || !(inv_temperature > 0.f && inv_temperature <= 3.4028235e38f)) return PNN_EINVAL;
    for (int f : {fz, fg})
        if (const int s = element_status(f)) return s;
    if (rows >= ((int64_t)1 << 31) || vocab >= ((int64_t)1 << 31)) return PNN_EUNSUPPORTED;
    if (rows == 0 || vocab == 0) return PNN_OK;
    if (!logits || !lse || !dlogits || (g_logprob && !targets) || (g_entropy && !entropy)) return PNN_EINVAL;
    discard_stale_hip_error();
    const LogprobBwd a = {logits, targets, lse, entropy, g_logprob, g_entropy, dlogits, vocab, ldz, ldg, inv_temperature, kind_of(fz), kind_of(fg), elem_fmt(fz), elem_fmt(fg)};
    hipLaunchKernelGGL(logprob_bwd_kernel, dim3((unsigned)rows), dim3(256), 0, (hipStream_t)stream, a);
    return hip_status(hipGetLastError());
}
