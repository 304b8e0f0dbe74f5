// posit_sample: one token for each row of logits, from a given random number.
//
// The order of the draw is that of falling logits, so what the limits leave is always the first of that order, and limits and draw alike ask for the place where a running sum
// first reaches a number: of counts (top_k), or of weights (top_p, the draw).  No row is sorted for it: a row's logits are counted by the highest bits of their order, and
// the place is looked up in the sums over these; of the logits in the one part that holds it, the next bits are counted, until it is one value's.  Weights are integers (the largest 2^s), so that a sum
// is the same in any order and the result does not depend on the device's.
#include "../../include/positnn_generate.h"
#include "lm_codec.h"
#include "sample_bins.h"

namespace pnn {

struct Sample {
    const void* z;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t* top_k;
    int32_t *token, *kept;
    float* logprob;
    int64_t vocab, ldz;
    int shift;           // s
    ElemFmt f;
    int64_t row0;        // the launch's first row
    // Rows cut into parts: what the parts leave for the last kernel
    int parts;
    uint32_t* tops;              // [row][part]: the largest key, all ones where there is a NaN or +inf
    uint32_t* counts;            // [row][bins + 1]: the last one the number of at least min_p
    unsigned long long* weights; // [row][bins]
};

constexpr int SAMPLE_THREADS = 1024, SAMPLE_LIST = 512, SAMPLE_COPIES = 16;

struct SampleBins {
    uint32_t count[SAMPLE_BINS];     // sums from the first bin to each, behind sample_sums
    unsigned long long weight[SAMPLE_BINS];
};
struct SampleShared {
    SampleBins first, next;
    uint32_t wave_count[16];
    unsigned long long wave_weight[16];
    double powers[256];              // 2^(i / 256)
    ulonglong2 list[SAMPLE_LIST];    // place in the order (key, complement of the index) and weight
    uint4 run[SAMPLE_LIST][2];       // eight logits as they lie in memory
    int run_index[SAMPLE_LIST];
    int listed, runs;
    uint32_t found_before;
    unsigned long long found, found_weight, found_own;
};

// A place in the order: the value that it falls on, as its key, how many are in front of that value (of the logit itself where its index is known) and what they weigh, and how
// many have it
struct SamplePlace {
    uint32_t key, before, n;
    int index;  // or -1
    unsigned long long weight_before, own;  // own: a logit's, where its index is known
};

__device__ __forceinline__ uint32_t sample_up(uint32_t v, int by, int lane) {
    const uint32_t o = (uint32_t)__shfl_up((int)v, by, 64);
    return lane >= by ? o : 0u;
}
// The bins' counts and weights to sums; by all threads, behind a barrier and with one behind it
__device__ __forceinline__ void sample_sums(SampleShared& sh, SampleBins& b) {
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const uint32_t c0 = b.count[2 * t], c1 = b.count[2 * t + 1];
    const unsigned long long w0 = b.weight[2 * t], w1 = b.weight[2 * t + 1];
    uint32_t c = c0 + c1;
    unsigned long long s = w0 + w1;
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        c += sample_up(c, by, lane);
        s += (unsigned long long)sample_up((uint32_t)(s >> 32), by, lane) << 32 | sample_up((uint32_t)s, by, lane);
    }
    if (lane == 63) {
        sh.wave_count[w] = c;
        sh.wave_weight[w] = s;
    }
    __syncthreads();
    for (int o = 0; o < w; ++o) {
        c += sh.wave_count[o];
        s += sh.wave_weight[o];
    }
    b.count[2 * t] = c - c1;
    b.count[2 * t + 1] = c;
    b.weight[2 * t] = s - w1;
    b.weight[2 * t + 1] = s;
    __syncthreads();
}
__device__ __forceinline__ void sample_clear(SampleBins& b) {
    for (int i = threadIdx.x; i < SAMPLE_BINS; i += SAMPLE_THREADS) {
        b.count[i] = 0;
        b.weight[i] = 0;
    }
}
// The bin where the sums first reach `want`, which the last one does: 64 of them at a time by the lanes of each wave
template <class T>
__device__ __forceinline__ int sample_search(const T* sums, unsigned long long want) {
    const int lane = threadIdx.x & 63;
    const int run = __builtin_ctzll(__ballot(sums[lane * 32 + 31] >= want));
    return run * 32 + __builtin_ctzll(__ballot(sums[run * 32 + (lane & 31)] >= want));
}

// u times w rounded down or up, for 0 <= u < 1 and w < 2^62
__device__ __forceinline__ unsigned long long sample_share(float u, unsigned long long w, bool up) {
    const uint32_t b = bits_of_f32(u);
    const int e = (int)(b >> 23);
    if (e == 0) return up && b != 0 && w != 0 ? 1 : 0;  // below 2^-126
    const unsigned long long m = (b & 0x7FFFFFu) | 0x800000u;
    const unsigned __int128 p = (unsigned __int128)m * w;
    const int by = 150 - e;  // at least 24
    if (by >= 100) return up && p != 0 ? 1 : 0;
    unsigned long long r = (unsigned long long)(p >> by);
    if (up && (p & (((unsigned __int128)1 << by) - 1)) != 0) ++r;
    return r;
}

// 2^s exp((z - m) / temperature), and that rounded to a whole number.  As 2^(t / 256): the nearest whole number of t from a table and the exponent, the rest by the series of the
// exponential function, whose next term is below 2^-54 of the sum.
struct SampleWeight {
    double m, c;         // t = (z - m) c
    float lowest;        // from it down weights are less than a quarter of one, and count as its
    const double* powers;
    int shift;
    __device__ __forceinline__ double raw(float z) const {
        const double t = ((double)__builtin_amdgcn_fmed3f(z, lowest, 3.4028235e38f) - m) * c;
        const double k = t + 0x1.8p52;
        const int n = (int)__builtin_bit_cast(unsigned long long, k);
        constexpr double L = 0.0027076061740622863;  // ln 2 / 256
        const double r = t - (k - 0x1.8p52);
        const double q = r * fma(r, fma(r, fma(r, L * L * L * L / 24, L * L * L / 6), L * L / 2), L);
        const unsigned long long p = __builtin_bit_cast(unsigned long long, powers[n & 255]) + ((unsigned long long)(uint32_t)((n >> 8) + shift) << 52);
        const double f = __builtin_bit_cast(double, p);
        return fma(f, q, f);
    }
    // the sum's last bit is 1
    static __device__ __forceinline__ unsigned long long whole(double e) { return __builtin_bit_cast(unsigned long long, e + 0x1p52) & 0xFFFFFFFFFFFFFull; }
    __device__ __forceinline__ unsigned long long of(float z) const { return whole(raw(z)); }
};

// NC: vectors of eight logits that a thread holds in registers, so that memory is read once; 0: rows of any length, read again by each pass.
// SAMPLE_WHOLE: a row to a workgroup.  Few long rows would leave most of the chip without work, so they go in parts of 8 NC logits a thread: SAMPLE_TOPS finds the parts' largest, SAMPLE_PARTS
// counts and weighs them into the rows' first bins (sums of integers, the same in any order), SAMPLE_JOIN does the rest, a row to a workgroup.
// Bound by the weights in binary64 and the search's passes: 256 x 50021 posit<16,1>, all limits: loads and maximum 4 us, weights into the histogram 20, the three places 20; memory would take 5.
enum SamplePhase { SAMPLE_WHOLE, SAMPLE_TOPS, SAMPLE_PARTS, SAMPLE_JOIN };

template <int K, int NC, int PHASE>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(Sample a) {
    constexpr bool POSIT = K == KIND_POSIT_U8 || K == KIND_POSIT_U16;
    constexpr int KEY = K == KIND_POSIT_U8 ? 8 : (K == KIND_F32 ? 32 : 16);  // bits of a key
    constexpr int FIRST = KEY < SAMPLE_BITS ? KEY : SAMPLE_BITS, DOWN = KEY - FIRST;
    __shared__ SampleShared sh;
    __shared__ uint32_t part[16];
    const int t = threadIdx.x;
    constexpr bool PART = PHASE == SAMPLE_TOPS || PHASE == SAMPLE_PARTS;
    const unsigned nth = PART ? blockIdx.x / (unsigned)a.parts : blockIdx.x, piece = PART ? blockIdx.x - nth * a.parts : 0;
    const int64_t row = a.row0 + nth, begin = (int64_t)piece * (NC * SAMPLE_THREADS * 8);
    const int n = PART && a.vocab - begin > NC * SAMPLE_THREADS * 8 ? NC * SAMPLE_THREADS * 8 : (int)(a.vocab - begin);  // of the row, or of the part
    const float inf = f32_of_bits(0x7F800000u), nan = f32_of_bits(0x7FC00000u);

    constexpr int W = K == KIND_POSIT_U8 ? 2 : (K == KIND_F32 ? 8 : 4), B = W / 2;  // words of eight logits, bytes of one
    struct Eight {
        uint32_t w[W];
    };
    const char* const src = (const char*)a.z + (row * a.ldz + begin) * B;
    // at the row's end the last logits again, of which only the `left` first places count
    auto load = [&](Eight& r, int64_t i) {
        if (i + 8 <= n) {
            __builtin_memcpy(r.w, src + i * B, 4 * W);
            return;
        }
        uint32_t x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t j = i + e < n ? i + e : n - 1;
            x[e] = B == 1 ? ((const uint8_t*)src)[j] : B == 2 ? ((const uint16_t*)src)[j] : ((const uint32_t*)src)[j];
        }
#pragma unroll
        for (int y = 0; y < W; ++y) r.w[y] = B == 1 ? x[(4 * y) & 7] | x[(4 * y + 1) & 7] << 8 | x[(4 * y + 2) & 7] << 16 | x[(4 * y + 3) & 7] << 24 : B == 2 ? x[(2 * y) & 7] | x[(2 * y + 1) & 7] << 16 : x[y];
    };
    constexpr int MANY = K == KIND_F32 ? 2 : 4;
    constexpr int STEP = SAMPLE_THREADS * 8, AT_ONCE = NC > 0 ? NC : 4;
    Eight held[AT_ONCE] = {};
    if (NC > 0) {
#pragma unroll
        for (int x = 0; x < AT_ONCE; ++x)
            if (t * 8 + x * STEP < n) load(held[x], t * 8 + x * STEP);
    }
    // every vector of the thread: f(words, their first index, how many)
    auto vectors = [&](auto f) {
        if (NC > 0) {
#pragma unroll
            for (int x = 0; x < AT_ONCE; ++x) {
                const int i = t * 8 + x * STEP;
                // words anew for each pass: what one works out of them is not kept for the next, for which there are no registers
#pragma unroll
                for (int y = 0; y < W; ++y) asm volatile("" : "+v"(held[x].w[y]));
                if (i < n) f(held[x], i, n - i);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            for (int64_t i0 = t * 8; i0 < n; i0 += AT_ONCE * STEP) {
#pragma unroll
                for (int x = 0; x < AT_ONCE; ++x)
                    if (i0 + x * STEP < n) load(held[x], i0 + x * STEP);
#pragma unroll
                for (int x = 0; x < AT_ONCE; ++x)
                {
                    if (i0 + x * STEP < n) f(held[x], (int)(i0 + x * STEP), (int)(n - (i0 + x * STEP)));
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    };
    auto element = [&](const Eight& r, int e) -> uint32_t { return B == 4 ? r.w[e % W] : (r.w[e * B / 4 % W] >> (8 * B * (e % (4 / (B < 4 ? B : 2))))) & (B == 1 ? 0xFFu : 0xFFFFu); };
    // the order of logits as integers; 0 and what is at or below NONE is never drawn
    auto key_of = [&](uint32_t x) -> uint32_t {
        if (K == KIND_POSIT_U8) return x ^ 0x80u;
        if (K == KIND_POSIT_U16) return ((x << (16 - a.f.n)) ^ 0x8000u) & 0xFFFFu;
        const uint32_t b = bits_of_f32(value_of<K>(x, a.f) + 0.f), o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
        return K == KIND_BF16 ? o >> 16 : o;
    };
    auto value_of_key = [&](uint32_t key) -> float {
        if (K == KIND_POSIT_U8) return posit_value(key ^ 0x80u, a.f);
        if (K == KIND_POSIT_U16) return posit_value((key ^ 0x8000u) >> (16 - a.f.n), a.f);
        const uint32_t o = K == KIND_BF16 ? key << 16 : key, b = o & 0x80000000u ? o ^ 0x80000000u : ~o;
        return f32_of_bits(K == KIND_BF16 ? b & 0xFFFF0000u : b);
    };
    constexpr uint32_t NONE = POSIT ? 0u : (K == KIND_BF16 ? 0x007Fu : 0x007FFFFFu);  // -inf

    uint32_t top = 0;
    bool bad = false;
    if (PHASE == SAMPLE_PARTS || PHASE == SAMPLE_JOIN) {
        for (int i = t; i < a.parts; i += SAMPLE_THREADS) {
            const uint32_t k = a.tops[row * a.parts + i];
            bad |= k == ~0u;
            top = k > top ? k : top;
        }
    } else vectors([&](const Eight& r, int, int) {  // the last logit again does no harm here
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t x = element(r, e), k = key_of(x);
            if (POSIT) bad |= k == 0u;
            else bad |= !(value_of<K>(x, a.f) < inf);
            top = k > top ? k : top;
        }
    });
    top = wave_max_u32(top);
    if ((t & 63) == 0) part[t >> 6] = top;
    if (t < 256) sh.powers[t] = exp2((double)t * (1.0 / 256));
    if (t == 0) {
        sh.found = sh.found_weight = sh.found_own = 0;
        sh.found_before = 0;
    }
    sample_clear(sh.first);
    if (K == KIND_POSIT_U8) sample_clear(sh.next);  // the copies
    bad = __syncthreads_or(bad);
    for (int w = 0; w < 16; ++w) top = part[w] > top ? part[w] : top;

    if (PHASE == SAMPLE_TOPS) {
        if (t == 0) a.tops[row * a.parts + piece] = bad ? ~0u : top;
        for (int i = piece * SAMPLE_THREADS + t; i <= SAMPLE_BINS; i += a.parts * SAMPLE_THREADS) {
            a.counts[row * (SAMPLE_BINS + 1) + i] = 0;
            if (i < SAMPLE_BINS) a.weights[row * SAMPLE_BINS + i] = 0;
        }
        return;
    }
    const float temp = a.temperature ? a.temperature[row] : 1.f;
    if (bad || top <= NONE || !(temp >= 0.f)) {
        if (PHASE != SAMPLE_PARTS && t == 0) {
            a.token[row] = -1;
            if (a.logprob) a.logprob[row] = bad || !(temp >= 0.f) ? nan : -inf;
            if (a.kept) a.kept[row] = 0;
        }
        return;
    }
    const bool greedy = temp == 0.f;
    const double m = (double)value_of_key(top), inverse = greedy ? 0.0 : 1.0 / (double)temp, unit = (double)((unsigned long long)1 << a.shift);
    // (s + 3) ln 2 temperatures below the largest, or the next number below that; where numbers are so far apart that this is hundreds of temperatures, c is less, which
    // leaves a weight of nothing one that the exponent can hold
    const double from = m - (a.shift + 3) * 0.6931471805599453 * (double)temp;
    float lowest = from > -3.4028234663852886e38 ? (float)from : -3.4028235e38f;
    if ((double)lowest > from || (double)lowest >= m) lowest = nextafterf(lowest, -inf);
    if (greedy || !(lowest > -inf)) lowest = -3.4028235e38f;
    const double c = inverse * (256 * 1.4426950408889634), most = 256.0 * 900.0 / (m - (double)lowest);
    const SampleWeight weight = {m, c < most || m == (double)lowest ? c : most, lowest, sh.powers, a.shift};
    float least = a.min_p ? a.min_p[row] : 0.f;
    least = least > 1.f ? 1.f : (least > 0.f ? least : 0.f);
    const double likely_from = (double)least * unit < 0.25 ? 0.0 : (double)least * unit;
    uint32_t likely = 0;  // of at least min_p
    // The first bins: of posits a key's highest bits, of floats the difference to the largest in steps of 1/2048 of the range whose weights are not nothing (a float's highest bits would
    // leave thousands in a bin); -inf is in none
    const float mf = (float)m, scale = sample_bin_scale(a.shift, inverse, greedy);
    auto bin_of = [&](uint32_t key, float v) -> int { return POSIT ? (int)((key ^ ((1u << KEY % 32) - 1u)) >> DOWN) : sample_float_bin(v, mf, scale); };
    if (PHASE == SAMPLE_JOIN) {
        for (int i = t; i < SAMPLE_BINS; i += SAMPLE_THREADS) {
            sh.first.count[i] = a.counts[row * (SAMPLE_BINS + 1) + i];
            sh.first.weight[i] = a.weights[row * SAMPLE_BINS + i];
        }
        __syncthreads();
    } else if (K == KIND_POSIT_U8) {
        // 256 values at most: counts alone, 16 copies of each for the lanes of a wave to meet fewer conflicts, and a weight each
        uint32_t* const copies = (uint32_t*)&sh.next;
        vectors([&](const Eight& r, int, int left) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) atomicAdd(&copies[(255u - key_of(element(r, e))) * SAMPLE_COPIES + (t & (SAMPLE_COPIES - 1))], 1u);
        });
        __syncthreads();
        if (t < 256) {
            uint32_t count = 0;
            for (int c = 0; c < SAMPLE_COPIES; ++c) count += copies[t * SAMPLE_COPIES + ((c + t) & (SAMPLE_COPIES - 1))];
            const double e = count ? weight.raw(value_of_key(255u - t)) : 0.0;
            sh.first.count[t] = count;
            sh.first.weight[t] = count * SampleWeight::whole(e);
            likely = e >= likely_from ? count : 0;
        }
    } else {
        const bool some = a.min_p != nullptr;
        auto add = [&](uint32_t x, float v) {
            // -inf is not counted: most of a row may be, and all of it in one bin
            const double e = weight.raw(v);
            const int bin = bin_of(POSIT ? key_of(x) : 0u, v);
            if (POSIT || bin >= 0) {
                atomicAdd(&sh.first.count[bin], 1u);
                atomicAdd(&sh.first.weight[bin], SampleWeight::whole(e));
                if (some) likely += e >= likely_from ? 1 : 0;
            }
        };
        vectors([&](const Eight& r, int, int left) {
            if (left < 8) return;
            Raw8 raw;
#pragma unroll
            for (int y = 0; y < W; ++y) raw.w[y] = r.w[y];
            float v[8];
            values8(v, raw, K, a.f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                add(element(r, e), v[e]);
                if (e % (NC > MANY ? 2 : 4) == (NC > MANY ? 1 : 3)) __builtin_amdgcn_sched_barrier(0);  // more side by side would not fit the registers
            }
        });
        // behind the last whole vector a logit to a thread
        if (t < n % 8) {
            const int64_t i = n - n % 8 + t;
            const uint32_t x = B == 4 ? ((const uint32_t*)src)[i] : ((const uint16_t*)src)[i];
            add(x, value_of<K>(x, a.f));
        }
    }
    if (PHASE == SAMPLE_JOIN) {
        likely = a.counts[row * (SAMPLE_BINS + 1) + SAMPLE_BINS];
    } else {
        uint32_t sum = likely;
#define PNN_STEP(CTRL, ROWS) sum += lane_shift<CTRL, ROWS>(sum, 0u);
        PNN_STEP(0x111, 0xF) PNN_STEP(0x112, 0xF) PNN_STEP(0x114, 0xF) PNN_STEP(0x118, 0xF) PNN_STEP(0x142, 0xA) PNN_STEP(0x143, 0xC)
#undef PNN_STEP
        __syncthreads();  // part has been read
        if ((t & 63) == 63) part[t >> 6] = sum;
        __syncthreads();
        likely = 0;
        for (int w = 0; w < 16; ++w) likely += part[w];
    }
    if (PHASE == SAMPLE_PARTS) {
        for (int i = t; i < SAMPLE_BINS; i += SAMPLE_THREADS) {
            const uint32_t c = sh.first.count[i];
            const unsigned long long w = sh.first.weight[i];
            if (c) atomicAdd(&a.counts[row * (SAMPLE_BINS + 1) + i], c);
            if (w) atomicAdd(&a.weights[row * SAMPLE_BINS + i], w);
        }
        if (t == 0 && likely) atomicAdd(&a.counts[row * (SAMPLE_BINS + 1) + SAMPLE_BINS], likely);
        return;
    }
    sample_sums(sh, sh.first);
    const uint32_t all = sh.first.count[SAMPLE_BINS - 1];
    if (!a.min_p) likely = all;

    // vectors with a logit in the first bins' `bin`, so no more of them than logits that it counts: which of those in registers have one first, then one after the other, so that what is done with them stands here once
    auto has = [&](const Eight& r, int bin) -> bool {
        if (K == KIND_POSIT_U16) {
            // the patterns' bits in the place of the key's, two in a word: whether one is zero
            const int up = 16 - a.f.n;
            const uint32_t cut = ((0xFFFFu << (DOWN > up ? DOWN : up)) & 0xFFFFu) * 0x10001u, other = ((uint32_t)((1 << FIRST) - 1 - bin) << DOWN ^ 0x8000u) * 0x10001u;
            uint32_t none = 0x80008000u;
#pragma unroll
            for (int x = 0; x < W; ++x) {
                const uint32_t y = ((r.w[x] << up) ^ other) & cut;
                none &= ((y & 0x7FFF7FFFu) + 0x7FFF7FFFu) | y;
            }
            return (none & 0x80008000u) != 0x80008000u;
        }
        bool any = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) any |= bin_of(POSIT ? key_of(element(r, e)) : 0u, POSIT ? 0.f : value_of<K>(element(r, e), a.f)) == bin;
        return any;
    };
    auto those = [&](int bin, auto f) {
        for (int64_t i0 = t * 8; i0 < n; i0 += AT_ONCE * STEP) {
            uint32_t some = 0;
            if (NC == 0) {
#pragma unroll
                for (int x = 0; x < AT_ONCE; ++x)
                    if (i0 + x * STEP < n) load(held[x], i0 + x * STEP);
            }
#pragma unroll
            for (int x = 0; x < AT_ONCE; ++x) {
#pragma unroll
                for (int y = 0; y < W; ++y) asm volatile("" : "+v"(held[x].w[y]));
                some |= has(held[x], bin) && i0 + x * STEP < n ? 1u << x : 0u;
            }
#pragma nounroll
            while (some) {
                const int at = __builtin_ctz(some);
                some &= some - 1;
                Eight r = held[0];
#pragma unroll
                for (int x = 1; x < AT_ONCE; ++x)
#pragma unroll
                    for (int y = 0; y < W; ++y) r.w[y] = at == x ? held[x].w[y] : r.w[y];
                const int64_t i = i0 + at * STEP;
                f(r, (int)i, (int)(n - i));
            }
        }
    };
    auto in_bin = [&](uint32_t k, int bin) { return bin_of(k, POSIT ? 0.f : value_of_key(k)) == bin; };
    auto each_of = [&](const Eight& r, int left, int bin, auto f) {
#pragma nounroll
        for (int e = 0; e < 8 && e < left; ++e) {
            uint32_t x = 0;
#pragma unroll
            for (int y = 0; y < 8; ++y) x = e == y ? element(r, y) : x;
            const uint32_t k = key_of(x);
            if (in_bin(k, bin)) f(k, e);
        }
    };
    int listed = -1, last_bin = 0;  // the bin whose logits the list holds; that of the last place
    // where the sum of counts or weights first reaches `want`, which the whole sum does
    auto place = [&](bool by_count, unsigned long long want) -> SamplePlace {
        SamplePlace p;
        const int bin = by_count ? sample_search(sh.first.count, want) : sample_search(sh.first.weight, want);
        p.before = bin ? sh.first.count[bin - 1] : 0;
        p.weight_before = bin ? sh.first.weight[bin - 1] : 0;
        p.n = sh.first.count[bin] - p.before;
        p.index = -1;
        last_bin = bin;
        if (K == KIND_POSIT_U8) {
            p.key = (uint32_t)((1 << FIRST) - 1 - bin);
            return p;
        }
        if (p.n <= (uint32_t)SAMPLE_LIST) {
            // few logits: each finds its place among them, one of them the place that is looked for.  The list holds their vectors, too: each has one of the bin's logits at least.
            if (listed != bin) {
                __syncthreads();
                if (t == 0) sh.listed = sh.runs = 0;
                if (t < SAMPLE_LIST) sh.list[t] = make_ulonglong2(0, 0);
                __syncthreads();
                // vectors first, then an element of them to a thread: few lanes of a wave have one at the same time
                those(bin, [&](const Eight& r, int i, int) {
                    const int at = atomicAdd(&sh.runs, 1);
                    if (at < SAMPLE_LIST) {
                        sh.run_index[at] = i;
                        __builtin_memcpy(sh.run[at], r.w, 4 * W);
                    }
                });
                __syncthreads();
                const int runs = sh.runs < SAMPLE_LIST ? sh.runs : SAMPLE_LIST;
                for (int y = t; y < runs * 8; y += SAMPLE_THREADS) {
                    const int e = y & 7, i = sh.run_index[y >> 3] + e;
                    const char* const at = (const char*)sh.run[y >> 3];
                    const uint32_t x = B == 1 ? ((const uint8_t*)at)[e] : B == 2 ? ((const uint16_t*)at)[e] : ((const uint32_t*)at)[e], k = key_of(x);
                    if (i < n && in_bin(k, bin)) {
                        const int to = atomicAdd(&sh.listed, 1);
                        if (to < SAMPLE_LIST) sh.list[to] = make_ulonglong2((unsigned long long)k << 32 | (uint32_t)~i, weight.of(value_of_key(k)));
                    }
                }
                listed = bin;
            }
            __syncthreads();
            if (t < (int)p.n) {
                const ulonglong2 mine = sh.list[t];
                uint32_t c = p.before;
                unsigned long long s = p.weight_before;
                for (uint32_t j = 0; j < p.n; j += 4) {  // reads in flight; behind the list's end there are zeros
                    ulonglong2 o[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) o[y] = sh.list[j + y];
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        c += o[y].x > mine.x ? 1u : 0u;
                        s += o[y].x > mine.x ? o[y].y : 0ull;
                    }
                }
                if (by_count ? (unsigned long long)c + 1 == want : s < want && s + mine.y >= want) {
                    sh.found = mine.x;
                    sh.found_before = c;
                    sh.found_weight = s;
                    sh.found_own = mine.y;
                }
            }
            __syncthreads();
            p.key = (uint32_t)(sh.found >> 32);
            p.index = (int)~(uint32_t)sh.found;
            p.before = sh.found_before;
            p.weight_before = sh.found_weight;
            p.own = sh.found_own;
            p.n = 1;
            return p;
        }
        // the bits of their keys from the highest, of the logits whose bits so far are the same
        p.key = 0;
        for (int down = KEY; down > 0;) {
            const int bits = down < SAMPLE_BITS ? down : SAMPLE_BITS;
            __syncthreads();
            sample_clear(sh.next);
            __syncthreads();
            those(bin, [&](const Eight& r, int, int left) {
                each_of(r, left, bin, [&](uint32_t k, int) {
                    if (down < KEY && k >> down != p.key) return;
                    const int b = (1 << bits) - 1 - (int)((k >> (down - bits)) & ((1u << bits) - 1u));
                    atomicAdd(&sh.next.count[b], 1u);
                    atomicAdd(&sh.next.weight[b], weight.of(value_of_key(k)));
                });
            });
            __syncthreads();
            sample_sums(sh, sh.next);
            const int b = by_count ? sample_search(sh.next.count, want - p.before) : sample_search(sh.next.weight, want - p.weight_before);
            const uint32_t c = b ? sh.next.count[b - 1] : 0;
            p.n = sh.next.count[b] - c;
            p.before += c;
            p.weight_before += b ? sh.next.weight[b - 1] : 0;
            p.key = p.key << bits | (uint32_t)((1 << bits) - 1 - b);
            down -= bits;
        }
        return p;
    };
    auto weight_of = [&](uint32_t key) { return weight.of(value_of_key(key)); };

    // how many stay, and what they weigh: by top_k, then top_p, then min_p; then the draw.  One loop, so that the search is there once.
    uint32_t stay = all;
    unsigned long long total = sh.first.weight[SAMPLE_BINS - 1], want = 0;
    const int k = greedy ? 1 : (a.top_k ? a.top_k[row] : 0);
    const float p = a.top_p ? a.top_p[row] : 1.f;
    float u = a.u[row];
    u = u > 0.f ? (u < 1.f ? u : 0x1.fffffep-1f) : 0.f;
    SamplePlace at = {};
#pragma nounroll
    for (int stage = 0; stage < 4; ++stage) {
        bool by_count = false;
        if (stage == 0 || stage == 2) {
            const uint32_t to = stage == 2 ? likely : (k > 0 ? (uint32_t)k : all);
            if (to >= stay) continue;
            by_count = true;
            want = to;
        } else if (stage == 1) {
            if (!(p < 1.f) || stay <= 1) continue;
            want = p > 0.f ? sample_share(p, total, true) : 0;
            want = want < 1 ? 1 : want;
        } else {
            want = sample_share(u, total, false) + 1;
        }
        at = place(by_count, want);
        if (stage == 3) break;
        if (at.index >= 0) {
            stay = at.before + 1;
            total = at.weight_before + at.own;
            continue;
        }
        const unsigned long long w = weight_of(at.key), some = by_count ? want - at.before : (want - at.weight_before + w - 1) / w;
        stay = at.before + (uint32_t)some;
        total = at.weight_before + some * w;
    }
    int token = at.index;
    if (token < 0) {
        // the nth of the logits of that value, by the bits of their indices from the highest
        const unsigned long long w = weight_of(at.key);
        uint32_t nth = (uint32_t)((want - at.weight_before + w - 1) / w);
        token = 0;
        int down = 32 - __builtin_clz((unsigned)n);
        for (int known = 32; down > 0;) {
            const int bits = down < SAMPLE_BITS ? down : SAMPLE_BITS, next = down - bits;
            __syncthreads();
            sample_clear(sh.next);
            __syncthreads();
            those(last_bin, [&](const Eight& r, int first, int left) {
                each_of(r, left, last_bin, [&](uint32_t k, int e) {
                    const int i = first + e;
                    if (k != at.key) return;
                    if (known == 32 || i >> known == token) atomicAdd(&sh.next.count[(i >> next) & ((1 << bits) - 1)], 1u);
                });
            });
            __syncthreads();
            sample_sums(sh, sh.next);
            const int bin = sample_search(sh.next.count, nth);
            nth -= bin ? sh.next.count[bin - 1] : 0;
            token = token << bits | bin;
            known = down = next;
        }
    }
    if (t == 0) {
        a.token[row] = token;
        if (a.logprob) a.logprob[row] = (float)(((double)value_of_key(at.key) - m) * inverse - log((double)total / unit));
        if (a.kept) a.kept[row] = (int32_t)stay;
    }
}

// s: the sum of `vocab` weights of 2^s stays below 2^63
inline int sample_shift(int64_t vocab) {
    int bits = 0;
    while (((int64_t)1 << bits) < vocab) ++bits;
    return 62 - bits < 51 ? 62 - bits : 51;
}

// Logits of a part, 0: rows are taken whole.  Parts pay where rows are long and few: they spread the weights over the chip, for two launches more.  All limits, us whole and in parts:
// posit<16,1>: 1 x 20011 27 and 30, 1 x 32003 33 and 33, 1 x 50021 40 and 34, 32 x 50021 47 and 44, 128 x 50021 50 and 62, 1 x 131072 79 and 46, 64 x 100003 85 and 78, 128 x 131072 98 and 106; binary32:
// 1 x 20011 26 and 30, 1 x 32003 33 and 33, 8 x 20011 61 and 60, 1 x 50021 48 and 38, 32 x 50021, rows at temperature 0 among them, 276 and 209; bfloat16 between these.  So the 3 to 4 us of a single row of less than 32000 are lost.
// 8-bit posits are counted without weights, and whole is the faster as long as a row fits the registers: 1 x 20011 29 and 36, 32 x 50021 43 and 49, 1 x 131072 40 and 40, 64 x 100003 65 and 77; behind that
// 1 x 150001 53 and 47, 8 x 200003 89 and 80, 64 x 150001 100 and 108, 128 x 300007 173 and 212.
inline int64_t sample_part(int fz, int64_t rows, int64_t vocab) {
    const bool counted = kind_of(fz) == KIND_POSIT_U8;
    return vocab > (counted ? 131072 : 16384) && rows <= vocab / (counted ? 8192 : 1024) ? SAMPLE_THREADS * 8 : 0;
}

// Rows that fit the threads' registers, 32 words each, stay there.
template <int K>
void launch_sample(hipStream_t st, unsigned rows, const Sample& a) {
    constexpr int MOST = K == KIND_POSIT_U8 ? 16 : (K == KIND_F32 ? 4 : 8);
    const int64_t vectors = (a.vocab + SAMPLE_THREADS * 8 - 1) / (SAMPLE_THREADS * 8);
    const dim3 block(SAMPLE_THREADS);
    if (a.parts > 0) {
        hipLaunchKernelGGL((sample_kernel<K, 1, SAMPLE_TOPS>), dim3(rows * a.parts), block, 0, st, a);
        hipLaunchKernelGGL((sample_kernel<K, 1, SAMPLE_PARTS>), dim3(rows * a.parts), block, 0, st, a);
        if (vectors <= MOST) hipLaunchKernelGGL((sample_kernel<K, MOST, SAMPLE_JOIN>), dim3(rows), block, 0, st, a);
        else hipLaunchKernelGGL((sample_kernel<K, 0, SAMPLE_JOIN>), dim3(rows), block, 0, st, a);
    } else if (vectors <= 2) {
        hipLaunchKernelGGL((sample_kernel<K, 2, SAMPLE_WHOLE>), dim3(rows), block, 0, st, a);
    } else if (vectors <= MOST) {
        hipLaunchKernelGGL((sample_kernel<K, MOST, SAMPLE_WHOLE>), dim3(rows), block, 0, st, a);
    } else {
        hipLaunchKernelGGL((sample_kernel<K, 0, SAMPLE_WHOLE>), dim3(rows), block, 0, st, a);
    }
}

}  // namespace pnn

using namespace pnn;

extern "C" size_t posit_sample_workspace(int fz, int64_t rows, int64_t vocab) {
    if (element_status(fz) || rows <= 0 || vocab <= 0 || rows >= ((int64_t)1 << 31) || vocab >= ((int64_t)1 << 31)) return 0;
    const int64_t part = sample_part(fz, rows, vocab);
    if (part == 0) return 0;
    return (size_t)rows * (SAMPLE_BINS * 8 + (SAMPLE_BINS + 1 + (vocab + part - 1) / part) * 4);
}

extern "C" int posit_sample(void* stream, int fz, int64_t rows, int64_t vocab, const void* logits, int64_t ldz, const float* u, const float* temperature, const int32_t* top_k,
                            const float* top_p, const float* min_p, int32_t* token, float* logprob, int32_t* kept, void* workspace, size_t workspace_bytes) {
    if (rows < 0 || vocab < 0 || ldz < vocab) return PNN_EINVAL;
    if (const int s = element_status(fz)) return s;
    if (vocab >= ((int64_t)1 << 31) || rows >= ((int64_t)1 << 31)) return PNN_EUNSUPPORTED;
    if (rows == 0 || vocab == 0) return PNN_OK;
    if (!logits || !u || !token) return PNN_EINVAL;
    const size_t need = posit_sample_workspace(fz, rows, vocab);
    if (need > 0 && (!workspace || workspace_bytes < need)) return PNN_EWORKSPACE;
    if (need > 0 && !aligned(workspace, 16)) return PNN_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    discard_stale_hip_error();
    Sample a = {logits, u, temperature, top_p, min_p, top_k, token, kept, logprob, vocab, ldz, sample_shift(vocab), elem_fmt(fz), 0, 0, nullptr, nullptr, nullptr};
    if (const int64_t part = sample_part(fz, rows, vocab)) {
        a.parts = (int)((vocab + part - 1) / part);
        a.weights = (unsigned long long*)workspace;
        a.counts = (uint32_t*)(a.weights + rows * SAMPLE_BINS);
        a.tops = a.counts + rows * (SAMPLE_BINS + 1);
    }
    for (const int64_t most = most_workgroups(SAMPLE_THREADS) / (a.parts > 0 ? a.parts : 1); a.row0 < rows; a.row0 += most) {
        const unsigned n = (unsigned)(rows - a.row0 < most ? rows - a.row0 : most);
        PNN_DISPATCH_KIND(kind_of(fz), launch_sample<K>(st, n, a))
    }
    return hip_status(hipGetLastError());
}
