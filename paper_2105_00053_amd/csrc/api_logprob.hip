// posit_token_logprob_fwd / posit_token_logprob_bwd: log probabilities of given tokens, entropy, top alternatives, and the gradient.
//
// Forward.  A workgroup takes a row, or a part of one where rows are few or long, into registers (64 words a thread) and goes
// over it there: maximum, then the sums of e^(z-m) and of e^(z-m) (z-m), then the alternatives; memory is read once.  A second kernel joins parts.
//  - 8-bit posits: 256 values at most, so a row is its histogram (in LDS, 16 copies of each bin, so that the lanes of a wave meet
//    few conflicts) and the sums are over 256 bins: no decoding, no exponential per logit; the k-th largest value is there too.
//  - 16-bit posits: the order of posits is that of their patterns as integers, so maximum and NaR come from packed integer instructions.
// Alternatives.  Each thread's largest logit (with the place of its vector) is sorted among the 256: the k-th largest of these
// bounds the k-th largest of all from below, and few logits are above it (about k + k^2 / 512 for random ones).  Those are collected and ranked by
// counting.  Where more are above it than the list holds, k rounds of a maximum take its place.
// What bounds it: the launch where rows are few (one of 100003 16-bit posits, 20 alternatives: 9 us and 7 for the join of 49 parts), an atomic addition in
// LDS a logit of 8 bits (2048 rows of 50021, 8 alternatives: 39 to 41 us for 102 MB, 2.5 TB/s; LDS 27 % of the cycles, nearly half of it conflicts, waves waiting 43 %), the
// vector unit's decoding and exponentials for 16 bits (4096 rows of 32000: 95 to 107 us for 262 MB, 2.6 TB/s; vector unit 85 %).  bfloat16 65 to 71 us, binary32 104 to 110 and 8 for the join.
#include "lm_codec.h"

namespace pnn {

typedef unsigned long long lp_key;  // order of the value in the high word, complement of the index in the low one: unique, 0 for none

struct LogprobFwd {
    const void* z;
    const int32_t* target;
    float *logprob, *lse, *entropy, *top_logprob;
    int32_t* top_index;
    int64_t vocab, ldz;
    float tau;
    int top, kind;
    ElemFmt f;
    int64_t row0;        // the launch's first row
    int64_t span;        // logits of a part, a multiple of 2048
    int parts;
    float4* part_stats;  // for more than one part: maximum, two sums, "holds a NaN or +inf"
    lp_key* part_keys;
};

constexpr float LP_LOG2E = 1.4426950408889634f;

// Order of binary32 values as integers, -0 as +0; that of posits is the pattern's.  -inf and what is below it is never an alternative.
__device__ __forceinline__ uint32_t lp_order(float v) {
    const uint32_t b = bits_of_f32(v + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
constexpr uint32_t LP_ORDER_OF_MINUS_INF = 0x007FFFFFu;
__device__ __forceinline__ uint32_t lp_order_posit(uint32_t p, ElemFmt f) { return (uint32_t)((int32_t)(p << (32 - f.n)) >> (32 - f.n)) ^ 0x80000000u; }
__device__ __forceinline__ float lp_value(uint32_t order, int kind, ElemFmt f) {
    if (kind == KIND_POSIT_U8 || kind == KIND_POSIT_U16) return posit_value((order ^ 0x80000000u) & ((1u << f.n) - 1u), f);
    return f32_of_bits(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}

constexpr int LP_LIST = 1024, LP_COPIES = 16;
struct LogprobTop {
    lp_key sorted[4][64];
    lp_key list[LP_LIST];
    lp_key result[64];
    lp_key bound;
    int count;
};

// The key of lane ^ MASK.  Through the vector unit where its lane shifts reach (a shuffle through LDS takes many times as long).
template <int MASK>
__device__ __forceinline__ uint32_t lp_swap32(uint32_t v) {
    if constexpr (MASK == 1) return lane_shift<0xB1, 0xF>(v, 0u);
    else if constexpr (MASK == 2) return lane_shift<0x4E, 0xF>(v, 0u);
    else if constexpr (MASK == 3) return lane_shift<0x1B, 0xF>(v, 0u);
    else if constexpr (MASK == 4) return lp_swap32<3>(lp_swap32<7>(v));
    else if constexpr (MASK == 7) return lane_shift<0x141, 0xF>(v, 0u);
    else if constexpr (MASK == 8) return lane_shift<0x128, 0xF>(v, 0u);
    else if constexpr (MASK == 15) return lane_shift<0x140, 0xF>(v, 0u);
    else return (uint32_t)__shfl_xor((int)v, MASK, 64);
}
template <int MASK>
__device__ __forceinline__ lp_key lp_swap(lp_key v) { return (lp_key)lp_swap32<MASK>((uint32_t)(v >> 32)) << 32 | lp_swap32<MASK>((uint32_t)v); }

// One step of sorting a wave's keys, the largest to the lowest lane: of lane and lane ^ MASK, the one without TOP (MASK's highest bit) keeps the larger.
template <int MASK, int TOP>
__device__ __forceinline__ lp_key lp_step(lp_key v) {
    const lp_key o = lp_swap<MASK>(v);
    const bool first = (threadIdx.x & TOP) == 0;
    return first == (v > o) ? v : o;
}
__device__ __forceinline__ lp_key lp_sort(lp_key v) {
    v = lp_step<1, 1>(v);
    v = lp_step<1, 1>(lp_step<3, 2>(v));
    v = lp_step<1, 1>(lp_step<2, 2>(lp_step<7, 4>(v)));
    v = lp_step<1, 1>(lp_step<2, 2>(lp_step<4, 4>(lp_step<15, 8>(v))));
    v = lp_step<1, 1>(lp_step<2, 2>(lp_step<4, 4>(lp_step<8, 8>(lp_step<31, 16>(v)))));
    return lp_step<1, 1>(lp_step<2, 2>(lp_step<4, 4>(lp_step<8, 8>(lp_step<16, 16>(lp_step<63, 32>(v))))));
}

// A bound from below for the k-th largest key of a workgroup, in sh.bound behind the next barrier (0: none).  `best`: each thread's largest, or a key that
// one of its own, at most `slack` below it, has.
__device__ __forceinline__ void lp_bound(LogprobTop& sh, lp_key best, uint32_t slack, int k) {
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    best = lp_sort(best);
    sh.sorted[w][lane] = best;
    __syncthreads();
    int at[3] = {0, 0, 0};  // keys of the other waves that are larger; all reads are issued, so that the three searches' latencies overlap
#pragma unroll
    for (int step = 64; step >= 1; step /= 2)
#pragma unroll
        for (int o = 0; o < 3; ++o) {
            const int to = at[o] + step, x = to <= 64 ? to - 1 : 63;
            at[o] = (sh.sorted[(w + o + 1) & 3][x] > best) & (to <= 64) ? to : at[o];
        }
    const int rank = lane + at[0] + at[1] + at[2];
    if (rank == k - 1 && best != 0) sh.bound = best - slack;
}

// The k largest keys of a workgroup, in order, in sh.result (0 where there are no more), given sh.bound; visit(bound, f) calls f with the thread's keys from
// `bound` up.
template <class Visit>
__device__ __forceinline__ void lp_select(LogprobTop& sh, int k, Visit visit) {
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    __syncthreads();
    const lp_key bound = sh.bound;
    visit(bound, [&](lp_key key) {
        const int n = atomicAdd(&sh.count, 1);
        if (n < LP_LIST) sh.list[n] = key;
    });
    __syncthreads();
    const int count = sh.count;
    if (count <= LP_LIST) {
        for (int i = t; i < count; i += 256) {
            const lp_key key = sh.list[i];
            int r = 0;
            for (int j = 0; j < count && r < k; j += 8)  // eight reads in flight; the list's length is a multiple of 8
#pragma unroll
                for (int x = 0; x < 8; ++x) r += (sh.list[j + x] > key) & (j + x < count) ? 1 : 0;
            if (r < k) sh.result[r] = key;
        }
    } else {
        lp_key last = ~0ull;
        for (int r = 0; r < k; ++r) {
            lp_key b = 0;
            visit(0, [&](lp_key key) { b = key < last && key > b ? key : b; });
#pragma unroll
            for (int m = 32; m >= 1; m >>= 1) {
                const lp_key o = (lp_key)(uint32_t)__shfl_xor((int)(uint32_t)(b >> 32), m, 64) << 32 | (uint32_t)__shfl_xor((int)(uint32_t)b, m, 64);
                b = o > b ? o : b;
            }
            __syncthreads();
            if (lane == 0) sh.sorted[w][0] = b;
            __syncthreads();
            for (int o = 0; o < 4; ++o) b = sh.sorted[o][0] > b ? sh.sorted[o][0] : b;
            if (t == 0) sh.result[r] = b;
            last = b;
            if (b == 0) break;
        }
    }
    __syncthreads();
}
// before lp_bound, with a barrier between
__device__ __forceinline__ void lp_clear(LogprobTop& sh) {
    if (threadIdx.x < 64) sh.result[threadIdx.x] = 0;
    if (threadIdx.x == 0) {
        sh.bound = 0;
        sh.count = 0;
    }
}

// A workgroup's maximum, and two of its sums; each once in a kernel, in words of `part` (12) of its own.
__device__ __forceinline__ float lp_block_max(float v, float* part) {
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}
__device__ __forceinline__ void lp_block_sums(float& s, float& u, float* part) {
    s = wave_sum(s);
    u = wave_sum(u);
    if ((threadIdx.x & 63) == 0) {
        part[4 + (threadIdx.x >> 6)] = s;
        part[8 + (threadIdx.x >> 6)] = u;
    }
    __syncthreads();
    s = (part[4] + part[5]) + (part[6] + part[7]);
    u = (part[8] + part[9]) + (part[10] + part[11]);
}

// A row's outputs from its maximum m (of z'), sums and alternatives; by all threads.
__device__ __forceinline__ void lp_outputs(const LogprobFwd& a, int64_t r, float m, float s, float u, bool bad, const lp_key* top) {
    const float inf = f32_of_bits(0x7F800000u), nan = f32_of_bits(0x7FC00000u);
    const bool empty = m == -inf;
    const float logs = logf(s);
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[r] = bad ? nan : (empty ? -inf : m + logs);
        if (a.entropy) a.entropy[r] = bad ? nan : (empty ? 0.f : logs - u / s);
        if (a.logprob) {
            const int32_t y = a.target[r];
            float lp = 0.f;
            if (bad || y >= a.vocab) lp = nan;
            else if (y >= 0) lp = empty ? -inf : fmaf(load_value(a.z, r * a.ldz + y, a.kind, a.f), a.tau, -m) - logs;
            a.logprob[r] = lp;
        }
    }
    for (int k = threadIdx.x; k < a.top; k += 256) {
        const lp_key key = bad ? 0 : top[k];
        a.top_index[r * a.top + k] = key ? (int32_t)~(uint32_t)key : -1;
        a.top_logprob[r * a.top + k] = bad ? nan : (key ? fmaf(lp_value((uint32_t)(key >> 32), a.kind, a.f), a.tau, -m) - logs : -inf);
    }
}

typedef short lp_pair __attribute__((ext_vector_type(2)));

template <int K>
__global__ __launch_bounds__(256) void logprob_part_kernel(LogprobFwd a) {
    constexpr int B = sizeof(typename Raw<K>::T), W = 2 * B, NC = 64 / W;  // words of a vector of 8, vectors to a thread
    constexpr bool POSIT = K == KIND_POSIT_U8 || K == KIND_POSIT_U16;
    __shared__ float part[12];
    __shared__ LogprobTop sh;
    __shared__ uint32_t hist[K == KIND_POSIT_U8 ? 256 * LP_COPIES : 1];
    const int t = threadIdx.x;
    const unsigned nth = blockIdx.x / (unsigned)a.parts;
    const int64_t row = a.row0 + nth;
    const int p = blockIdx.x - nth * a.parts;
    const int64_t begin = p * a.span;
    const int n = (int)(a.vocab - begin < a.span ? a.vocab - begin : a.span), vectors = n / 8, rest = n - vectors * 8;
    const char* const src = (const char*)a.z + (row * a.ldz + begin) * B;
    const float inf = f32_of_bits(0x7F800000u);
    lp_clear(sh);
    uint32_t raw[NC][W];
#pragma unroll
    for (int c = 0; c < NC; ++c)
        if (c * 256 + t < vectors) __builtin_memcpy(raw[c], src + (int64_t)(c * 256 + t) * 8 * B, 8 * B);
    // what is left behind the last whole vector: one logit to each of the first threads
    const bool extra = t < rest;
    uint32_t one = 0;
    if (extra) one = B == 1 ? ((const uint8_t*)src)[vectors * 8 + t] : B == 2 ? ((const uint16_t*)src)[vectors * 8 + t] : ((const uint32_t*)src)[vectors * 8 + t];
    if (K == KIND_POSIT_U8) {
#pragma unroll
        for (int c = 0; c < LP_COPIES / 4; ++c) ((uint4*)hist)[c * 256 + t] = make_uint4(0, 0, 0, 0);
        __syncthreads();
    }

    auto element = [&](const uint32_t* w, int e) -> uint32_t { return B == 4 ? w[e] : (w[e * B / 4] >> (8 * B * (e % (4 / B)))) & (B == 1 ? 0xFFu : 0xFFFFu); };
    // 16-bit posits: NaR, which is looked for by itself, comes out as zero here
    auto value = [&](uint32_t x) -> float {
        if (K != KIND_POSIT_U16) return value_of<K>(x, a.f);
        uint32_t y;
        const float v = posit_value_regular(x, a.f, y);
        return y == 0u ? 0.f : v;
    };
    auto order = [&](uint32_t x) -> uint32_t { return POSIT ? lp_order_posit(x, a.f) : lp_order(value(x)); };
    // the largest of a vector, as its order; for 16-bit posits the smallest too (NaR is the smallest of all)
    lp_pair least = {0, 0};
    auto vector_top = [&](const uint32_t* w, bool low) -> uint32_t {
        if constexpr (POSIT) {
            const int shift = 16 - a.f.n;  // patterns of 10 and 12 bits to the top of their half words
            lp_pair m;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                lp_pair x, y;
                if (B == 1) {
                    x = __builtin_bit_cast(lp_pair, w[i] & 0xFF00FF00u);
                    y = __builtin_bit_cast(lp_pair, (w[i] << 8) & 0xFF00FF00u);
                    x = __builtin_elementwise_max(x, y);
                } else {
                    x = __builtin_bit_cast(lp_pair, w[i]) << (short)shift;
                    if (low) least = __builtin_elementwise_min(least, x);
                }
                m = i ? __builtin_elementwise_max(m, x) : x;
            }
            const int v = m.x > m.y ? m.x : m.y;
            return (uint32_t)(v >> (B == 1 ? 8 : shift)) ^ 0x80000000u;
        } else {
            float m = value(element(w, 0));
#pragma unroll
            for (int e = 1; e < 8; ++e) m = fmaxf(m, value(element(w, e)));
            return m == m ? lp_order(m) : 0u;
        }
    };

    // each thread's largest, with the place of its vector
    uint32_t best = 0;
    int at = 0;
    auto look = [&](bool low) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (c * 256 + t >= vectors) continue;
            const uint32_t v = vector_top(raw[c], low);
            if (v > best) {
                best = v;
                at = (c * 256 + t) * 8;
            }
        }
        if (extra) {
            const uint32_t v = order(one);
            if (v > best) {
                best = v;
                at = vectors * 8 + t;
            }
        }
    };
    bool bounded = false;  // the histogram knows the k-th largest
    float m, s = 0.f, u = 0.f;
    bool bad = false;
    if (K == KIND_POSIT_U8) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (c * 256 + t >= vectors) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) atomicAdd(&hist[element(raw[c], e) * LP_COPIES + (t & (LP_COPIES - 1))], 1u);
        }
        if (extra) atomicAdd(&hist[one * LP_COPIES + (t & (LP_COPIES - 1))], 1u);
        __syncthreads();
        // thread t is bin t
        uint32_t count = 0;
#pragma unroll
        for (int c = 0; c < LP_COPIES / 4; ++c) {
            const uint4 x = ((const uint4*)hist)[t * (LP_COPIES / 4) + ((c + t) & (LP_COPIES / 4 - 1))];
            count += x.x + x.y + x.z + x.w;
        }
        const bool nar = t == 128;
        const float v = nar ? 0.f : posit_value(t, a.f) * a.tau;
        bad = __syncthreads_or(nar && count > 0);
        m = lp_block_max(count > 0 && !nar ? v : -inf, part);
        const float d = v - m, e = count > 0 ? (float)count * __builtin_amdgcn_exp2f(d * LP_LOG2E) : 0.f;
        s = e;
        u = e > 0.f ? e * d : 0.f;
        lp_block_sums(s, u, part);
        if (a.top > 0) {
            // logits in the bins from the largest value down to thread t's, 127 - t for what is not negative: where they reach k is the bound
            uint32_t* const down = hist;
            down[(127 - t) & 255] = count;
            __syncthreads();
            const uint32_t mine = down[t];
            uint32_t sum = mine;
#define PNN_STEP(CTRL, ROWS) sum += lane_shift<CTRL, ROWS>(sum, 0u);
            PNN_STEP(0x111, 0xF) PNN_STEP(0x112, 0xF) PNN_STEP(0x114, 0xF) PNN_STEP(0x118, 0xF) PNN_STEP(0x142, 0xA) PNN_STEP(0x143, 0xC)
#undef PNN_STEP
            if ((t & 63) == 63) down[256 + (t >> 6)] = sum;
            __syncthreads();
            for (int w = 0; w < (t >> 6); ++w) sum += down[256 + w];
            const bool here = sum >= (uint32_t)a.top && sum - mine < (uint32_t)a.top;
            if (here) sh.bound = (lp_key)lp_order_posit((uint32_t)(127 - t) & 0xFFu, a.f) << 32;
            bounded = !__syncthreads_or(here && sum > (uint32_t)LP_LIST);  // too many of that value for the list
            if (!bounded && t == 0) sh.bound = 0;
        }
    } else {
        look(K == KIND_POSIT_U16);
        const uint32_t t0 = wave_max_u32(best);
        if (POSIT) bad = __syncthreads_or(least.x == -32768 || least.y == -32768 || (extra && one == 1u << (a.f.n - 1)));
        m = lp_block_max(t0 == 0 ? -inf : lp_value(t0, K, a.f) * a.tau, part);
        if (m > -inf) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (c * 256 + t >= vectors) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float d = fmaf(value(element(raw[c], e)), a.tau, -m), x = __builtin_amdgcn_exp2f(d * LP_LOG2E);
                    s += x;
                    u = fmaf(x, POSIT ? d : fmaxf(d, -200.f), u);
                }
            }
            if (extra) {
                const float d = fmaf(value(one), a.tau, -m), x = __builtin_amdgcn_exp2f(d * LP_LOG2E);
                s += x;
                u = fmaf(x, POSIT ? d : fmaxf(d, -200.f), u);
            }
            lp_block_sums(s, u, part);
            bad = bad || !(s == s) || m == inf;
        } else if (!POSIT) {
            // nothing but -inf, and NaN perhaps
            bool nan = extra && value(one) != value(one);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (c * 256 + t >= vectors) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) nan |= value(element(raw[c], e)) != value(element(raw[c], e));
            }
            bad = __syncthreads_or(nan);
        }
    }

    if (a.top > 0) {
        auto key_of = [&](uint32_t x, int i) -> lp_key {
            const uint32_t o = order(x);
            return !POSIT && o <= LP_ORDER_OF_MINUS_INF ? 0 : (lp_key)o << 32 | (uint32_t)~(uint32_t)(begin + i);
        };
        auto visit = [&](lp_key bound, auto f) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (c * 256 + t >= vectors) continue;
                if (vector_top(raw[c], false) < (uint32_t)(bound >> 32)) continue;
                if constexpr (B == 4) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const lp_key key = key_of(raw[c][e], (c * 256 + t) * 8 + e);
                        if (key != 0 && key >= bound) f(key);
                    }
                } else {
                    lp_key lo = raw[c][0] | (lp_key)raw[c][1] << 32, hi = B == 1 ? 0 : raw[c][B == 1 ? 0 : 2] | (lp_key)raw[c][B == 1 ? 0 : 3] << 32;
#pragma unroll 1
                    for (int e = 0; e < 8; ++e) {
                        if (B == 2 && e == 4) lo = hi;
                        const lp_key key = key_of((uint32_t)lo & (B == 1 ? 0xFFu : 0xFFFFu), (c * 256 + t) * 8 + e);
                        lo >>= 8 * B;
                        if (key != 0 && key >= bound) f(key);
                    }
                }
            }
            if (extra) {
                const lp_key key = key_of(one, vectors * 8 + t);
                if (key != 0 && key >= bound) f(key);
            }
        };
        if (!bounded) {
            if (K == KIND_POSIT_U8) look(false);
            const bool any = POSIT ? best != 0 : best > LP_ORDER_OF_MINUS_INF;
            __syncthreads();
            lp_bound(sh, any ? (lp_key)best << 32 | (uint32_t)~(uint32_t)(begin + at) : 0, 7, a.top);
        }
        lp_select(sh, a.top, visit);
    }
    if (a.parts == 1) {
        lp_outputs(a, row, m, s, u, bad, sh.result);
        return;
    }
    const int64_t slot = row * a.parts + p;
    if (t == 0) a.part_stats[slot] = make_float4(m, s, u, bad ? 1.f : 0.f);
    for (int k = t; k < a.top; k += 256) a.part_keys[slot * a.top + k] = sh.result[k];
}

// Parts of a row joined, one row to a workgroup.
__global__ __launch_bounds__(256) void logprob_join_kernel(LogprobFwd a) {
    __shared__ float part[12];
    __shared__ LogprobTop sh;
    const int64_t row = a.row0 + blockIdx.x;
    const int t = threadIdx.x;
    const float inf = f32_of_bits(0x7F800000u);
    const float4* const st = a.part_stats + row * a.parts;
    float m = -inf;
    bool bad = false;
    lp_clear(sh);
    for (int i = t; i < a.parts; i += 256) {
        m = fmaxf(m, st[i].x);
        bad |= st[i].w != 0.f;
    }
    bad = __syncthreads_or(bad);
    m = lp_block_max(m, part);
    float s = 0.f, u = 0.f;
    for (int i = t; i < a.parts; i += 256) {
        const float4 x = st[i];
        if (x.x == -inf) continue;
        const float d = x.x - m, f = __builtin_amdgcn_exp2f(d * LP_LOG2E);
        s = fmaf(f, x.y, s);
        if (f > 0.f) u = fmaf(f, fmaf(x.y, d, x.z), u);
    }
    lp_block_sums(s, u, part);
    if (a.top > 0) {
        const lp_key* const keys = a.part_keys + row * a.parts * a.top;
        const int64_t n = (int64_t)a.parts * a.top;
        lp_key best = 0;
        for (int64_t i = t; i < n; i += 256) best = keys[i] > best ? keys[i] : best;
        lp_bound(sh, best, 0, a.top);
        lp_select(sh, a.top, [&](lp_key bound, auto f) {
            for (int64_t i = t; i < n; i += 256)
                if (keys[i] != 0 && keys[i] >= bound) f(keys[i]);
        });
    }
    lp_outputs(a, row, m, s, u, bad, sh.result);
}

// ---- gradient ----

struct LogprobBwd {
    const void* z;
    const int32_t* target;
    const float *lse, *entropy, *g_lp, *g_ent;
    void* dz;
    int64_t rows, vocab, ldz, ldg;
    float tau;
    int kg;
    ElemFmt fz, fg;
    int64_t row0;  // the launch's first row
    int64_t span;
    int parts;
};

// A part of a row to a workgroup, vectors of 8 to a thread, the next one in flight.  Bound by the vector unit for 16-bit posits (93 % of the cycles: decoding, an
// exponential, rounding), with memory not far: 4096 rows of 32000 to bfloat16 117 to 131 us for 524 MB, 4.3 TB/s; from bfloat16 80 to 94, from binary32 139 to 142 for 786 MB.
template <int K>
__global__ __launch_bounds__(256) void logprob_bwd_kernel(LogprobBwd a) {
    const int t = threadIdx.x;
    const unsigned nth = blockIdx.x / (unsigned)a.parts;
    const int64_t row = a.row0 + nth;
    const int64_t begin = (int64_t)(blockIdx.x - nth * a.parts) * a.span, end = begin + a.span < a.vocab ? begin + a.span : a.vocab;
    const float inf = f32_of_bits(0x7F800000u), lse = a.lse[row];
    const int32_t y = a.g_lp ? a.target[row] : -1;
    const float gl = y < 0 ? 0.f : (y >= a.vocab ? f32_of_bits(0x7FC00000u) : a.g_lp[row]) * a.tau;
    const float ge = a.g_ent ? a.g_ent[row] * a.tau : 0.f, h = a.g_ent ? a.entropy[row] : 0.f;
    const bool empty = lse == -inf;
    Raw8 raw;
    int64_t j = begin + t * 8;
    auto left = [&](int64_t i) { return i < end ? (end - i < 8 ? (int)(end - i) : 8) : 0; };
    load8(raw, a.z, row * a.ldz + j, K, left(j));
    for (; j < end; j += 2048) {
        float v[8];
        values8(v, raw, K, a.fz);
        load8(raw, a.z, row * a.ldz + j + 2048, K, left(j + 2048));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // 2^32 p, taken back by a product: exp2 itself has no subnormal results
            const float lp = empty ? -inf : fmaf(v[e], a.tau, -lse), p = __builtin_amdgcn_exp2f(fmaf(lp, LP_LOG2E, 32.f)) * 0x1p-32f;
            // p (g_lp + g_H (log p + H)), where a probability of zero has no log; a row that is NaN stays so
            const float k = fmaf(ge, lp + h, gl);
            v[e] = p == 0.f ? gl * -0.f : -p * k;
        }
        if ((uint64_t)(y - j) < 8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += j + e == y ? gl : 0.f;
        }
        Raw8 out;
        raw8<false>(out, v, a.kg, a.fg);
        store8(a.dz, row * a.ldg + j, out, a.kg, left(j));
    }
}

// Logits of a part: what 256 threads hold in 64 words each, less where that leaves most of the chip without work.
inline int64_t logprob_span(int fz, int64_t rows, int64_t vocab) {
    int64_t span = 16 * 2048 * 2 / (int64_t)element_bytes(fz);
    // A row that fits one workgroup's registers stays whole: the second kernel costs more than the parts save (32 rows, five alternatives, us: 5003 logits in
    // binary32 8.0 and 11.9, 16384 in 16-bit posits 10.9 and 12.8, 50021 in 8-bit ones 14.0 and 14.6; only 32000 in 16-bit ones, 14.4 and 13.5, would gain from
    // parts, by less than a rule with a second border is worth).
    if (vocab <= span) return span;
    while (span > 2048 && rows * ((vocab + span - 1) / span) < 512) span /= 2;
    return span;
}

}  // namespace pnn

using namespace pnn;

extern "C" size_t posit_token_logprob_workspace(int fz, int64_t rows, int64_t vocab, int top) {
    if (element_status(fz) || rows <= 0 || vocab <= 0 || top < 0 || top > 64) return 0;
    const int64_t span = logprob_span(fz, rows, vocab), parts = (vocab + span - 1) / span;
    return parts > 1 ? (size_t)(rows * parts * (16 + 8 * top)) : 0;
}

extern "C" int posit_token_logprob_fwd(void* stream, int fz, int64_t rows, int64_t vocab, const void* logits, int64_t ldz, const int32_t* targets,
                                       float inv_temperature, int top, float* logprob, float* lse, float* entropy, float* top_logprob, int32_t* top_index,
                                       void* workspace, size_t workspace_bytes) {
    if (rows < 0 || vocab < 0 || ldz < vocab || top < 0 || !(inv_temperature > 0.f && inv_temperature <= 3.4028235e38f)) return PNN_EINVAL;
    if (const int s = element_status(fz)) return s;
    if (top > 64 || vocab >= ((int64_t)1 << 31) || rows >= ((int64_t)1 << 31)) return PNN_EUNSUPPORTED;
    if (rows == 0 || vocab == 0) return PNN_OK;
    if (!logits || (logprob && !targets) || (top > 0 && (!top_logprob || !top_index)) || (!logprob && !lse && !entropy && top == 0)) return PNN_EINVAL;
    const int64_t span = logprob_span(fz, rows, vocab), parts = (vocab + span - 1) / span;
    const size_t need = posit_token_logprob_workspace(fz, rows, vocab, top);
    if (need > 0 && (!workspace || workspace_bytes < need)) return PNN_EWORKSPACE;
    if (need > 0 && !aligned(workspace, 16)) return PNN_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    discard_stale_hip_error();
    LogprobFwd a = {logits, targets, logprob, lse, entropy, top_logprob, top_index, vocab, ldz, inv_temperature, top, kind_of(fz), elem_fmt(fz), 0, span, (int)parts,
                    (float4*)workspace, (lp_key*)((char*)workspace + rows * parts * 16)};
    for (const int64_t most = most_workgroups(256) / parts; a.row0 < rows; a.row0 += most) {
        const int64_t n = rows - a.row0 < most ? rows - a.row0 : most;
        PNN_DISPATCH_KIND(a.kind, hipLaunchKernelGGL(logprob_part_kernel<K>, dim3((unsigned)(n * parts)), dim3(256), 0, st, a))
        if (parts > 1) hipLaunchKernelGGL(logprob_join_kernel, dim3((unsigned)n), dim3(256), 0, st, a);
    }
    return hip_status(hipGetLastError());
}

extern "C" int posit_token_logprob_bwd(void* stream, int fz, int fg, int64_t rows, int64_t vocab, const void* logits, int64_t ldz, const int32_t* targets,
                                       float inv_temperature, const float* lse, const float* entropy, const float* g_logprob, const float* g_entropy,
                                       void* dlogits, int64_t ldg) {
    if (rows < 0 || vocab < 0 || ldz < vocab || ldg < vocab || !(inv_temperature > 0.f && inv_temperature <= 3.4028235e38f)) return PNN_EINVAL;
    for (int f : {fz, fg})
        if (const int s = element_status(f)) return s;
    if (vocab >= ((int64_t)1 << 31) || rows >= ((int64_t)1 << 31)) return PNN_EUNSUPPORTED;
    if (rows == 0 || vocab == 0) return PNN_OK;
    if (!logits || !lse || !dlogits || (g_logprob && !targets) || (g_entropy && !entropy)) return PNN_EINVAL;
    // four vectors to a thread keep the next load in flight; parts of one where rows are few
    const int64_t span = rows * ((vocab + 8191) / 8192) >= 1024 ? 8192 : 2048, parts = (vocab + span - 1) / span;
    hipStream_t st = (hipStream_t)stream;
    discard_stale_hip_error();
    LogprobBwd a = {logits, targets, lse, entropy, g_logprob, g_entropy, dlogits, rows, vocab, ldz, ldg, inv_temperature, kind_of(fg), elem_fmt(fz), elem_fmt(fg), 0, span, (int)parts};
    for (const int64_t most = most_workgroups(256) / parts; a.row0 < rows; a.row0 += most) {
        const int64_t n = rows - a.row0 < most ? rows - a.row0 : most;
        PNN_DISPATCH_KIND(kind_of(fz), hipLaunchKernelGGL(logprob_bwd_kernel<K>, dim3((unsigned)(n * parts)), dim3(256), 0, st, a))
    }
    return hip_status(hipGetLastError());
}
