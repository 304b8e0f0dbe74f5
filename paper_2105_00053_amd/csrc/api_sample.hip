// posit_sample: one token for each row of logits, from a given random number.
//
// The order of the draw is that of falling logits, so what the limits leave is always the first of that order, and limits and draw alike ask for the place where a running sum
// first reaches a number: of counts (top_k), or of weights (top_p, the draw).  No row is sorted for it: a row's logits are counted by the highest bits of their order, and
// the place is looked up in the sums over these; of the logits in the one part that holds it, the next bits are counted, until it is one value's.  Weights are integers (the largest 2^s), so that a sum
// is the same in any order and the result does not depend on the device's.
#include "../../include/positnn_generate.h"
#include "lm_codec.h"

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
};

constexpr int SAMPLE_THREADS = 1024, SAMPLE_BITS = 11, SAMPLE_BINS = 1 << SAMPLE_BITS, SAMPLE_LIST = 1024;

struct SampleBins {
    uint32_t count[SAMPLE_BINS];     // sums from the first bin to each, behind sample_sums
    unsigned long long weight[SAMPLE_BINS];
};
struct SampleShared {
    SampleBins first, next;
    uint32_t wave_count[16];
    unsigned long long wave_weight[16];
    int list[SAMPLE_LIST];
    int listed, token;
    int found;
};

// A place in the order: the value that it falls on, as its key, how many are in front of that value and what they weigh, and how many have it
struct SamplePlace {
    uint32_t key, before, n;
    unsigned long long weight_before;
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

// u times w rounded down, for 0 <= u < 1 and w < 2^62
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

template <int K>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(Sample a) {
    constexpr bool POSIT = K == KIND_POSIT_U8 || K == KIND_POSIT_U16;
    constexpr int KEY = K == KIND_POSIT_U8 ? 8 : (K == KIND_F32 ? 32 : 16);  // bits of a key
    constexpr int FIRST = KEY < SAMPLE_BITS ? KEY : SAMPLE_BITS;
    __shared__ SampleShared sh;
    __shared__ uint32_t part[16];
    const int t = threadIdx.x;
    const int64_t row = a.row0 + blockIdx.x;
    const int n = (int)a.vocab;
    const float inf = f32_of_bits(0x7F800000u), nan = f32_of_bits(0x7FC00000u);

    auto each = [&](auto f) {
        for (int64_t i = t * 8; i < n; i += SAMPLE_THREADS * 8) {
            const int left = n - i < 8 ? (int)(n - i) : 8;
            Raw8 r;
            load8(r, a.z, row * a.ldz + i, K, left);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) f(K == KIND_F32 ? r.w[e] : pattern8(r, e, K), (int)(i + e));
        }
    };
    // the order of logits as integers; 0 and what is at or below `none` is never drawn
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
    each([&](uint32_t x, int) {
        const uint32_t k = key_of(x);
        if (POSIT) bad |= k == 0u;
        else bad |= !(value_of<K>(x, a.f) < inf);
        top = k > top ? k : top;
    });
    top = wave_max_u32(top);
    if ((t & 63) == 0) part[t >> 6] = top;
    sample_clear(sh.first);
    if (t == 0) sh.listed = 0;
    bad = __syncthreads_or(bad);
    for (int w = 0; w < 16; ++w) top = part[w] > top ? part[w] : top;

    const float temp = a.temperature ? a.temperature[row] : 1.f;
    if (bad || top <= NONE || !(temp >= 0.f)) {
        if (t == 0) {
            a.token[row] = -1;
            if (a.logprob) a.logprob[row] = bad || !(temp >= 0.f) ? nan : -inf;
            if (a.kept) a.kept[row] = 0;
        }
        return;
    }
    const bool greedy = temp == 0.f;
    const double m = (double)value_of_key(top), inverse = greedy ? 0.0 : 1.0 / (double)temp, unit = (double)((unsigned long long)1 << a.shift);
    auto share = [&](float z) -> double { return exp(((double)z - m) * inverse); };
    // to nearest: the sum's last bit is 1
    auto whole = [&](double e) -> unsigned long long { return __builtin_bit_cast(unsigned long long, e * unit + 0x1p52) & 0xFFFFFFFFFFFFFull; };
    float least = a.min_p ? a.min_p[row] : 0.f;
    least = least > 1.f ? 1.f : (least > 0.f ? least : 0.f);
    int likely = 0;  // of at least min_p
    constexpr int DOWN = KEY - FIRST;
    each([&](uint32_t x, int) {
        const uint32_t k = key_of(x);
        if (k <= NONE) return;
        const double e = share(value_of<K>(x, a.f));
        const int bin = (1 << FIRST) - 1 - (int)(k >> DOWN);
        atomicAdd(&sh.first.count[bin], 1u);
        atomicAdd(&sh.first.weight[bin], whole(e));
        likely += e >= (double)least ? 1 : 0;
    });
    {
        uint32_t sum = (uint32_t)likely;
#define PNN_STEP(CTRL, ROWS) sum += lane_shift<CTRL, ROWS>(sum, 0u);
        PNN_STEP(0x111, 0xF) PNN_STEP(0x112, 0xF) PNN_STEP(0x114, 0xF) PNN_STEP(0x118, 0xF) PNN_STEP(0x142, 0xA) PNN_STEP(0x143, 0xC)
#undef PNN_STEP
        __syncthreads();  // part has been read
        if ((t & 63) == 63) part[t >> 6] = sum;
        __syncthreads();
        likely = 0;
        for (int w = 0; w < 16; ++w) likely += (int)part[w];
    }
    sample_sums(sh, sh.first);
    const uint32_t all = sh.first.count[(1 << FIRST) - 1];

    // where the sum of counts (BY_COUNT) or weights first reaches `want`, which the whole sum does
    auto search = [&](const SampleBins& b, bool by_count, unsigned long long want) -> int {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int bin = 2 * t + i;
            const unsigned long long before = bin == 0 ? 0 : (by_count ? b.count[bin - 1] : b.weight[bin - 1]), sum = by_count ? b.count[bin] : b.weight[bin];
            if (before < want && sum >= want) sh.found = bin;
        }
        __syncthreads();
        return sh.found;
    };
    auto place = [&](bool by_count, unsigned long long want) -> SamplePlace {
        SamplePlace p;
        int bin = search(sh.first, by_count, want);
        p.before = bin ? sh.first.count[bin - 1] : 0;
        p.weight_before = bin ? sh.first.weight[bin - 1] : 0;
        p.n = sh.first.count[bin] - p.before;
        p.key = (uint32_t)((1 << FIRST) - 1 - bin);
        // the next bits, of the logits whose bits so far are these
        for (int down = DOWN; down > 0;) {
            const int bits = down < SAMPLE_BITS ? down : SAMPLE_BITS;
            __syncthreads();
            sample_clear(sh.next);
            __syncthreads();
            each([&](uint32_t x, int) {
                const uint32_t k = key_of(x);
                if (k >> down != p.key || k <= NONE) return;
                const int bin = (1 << bits) - 1 - (int)((k >> (down - bits)) & ((1u << bits) - 1u));
                atomicAdd(&sh.next.count[bin], 1u);
                atomicAdd(&sh.next.weight[bin], whole(share(value_of<K>(x, a.f))));
            });
            __syncthreads();
            sample_sums(sh, sh.next);
            bin = search(sh.next, by_count, want - (by_count ? p.before : p.weight_before));
            const uint32_t c = bin ? sh.next.count[bin - 1] : 0;
            p.n = sh.next.count[bin] - c;
            p.before += c;
            p.weight_before += bin ? sh.next.weight[bin - 1] : 0;
            p.key = p.key << bits | (uint32_t)((1 << bits) - 1 - bin);
            down -= bits;
        }
        return p;
    };
    auto weight_of = [&](uint32_t key) { return whole(share(value_of_key(key))); };

    // how many stay, and what they weigh
    uint32_t stay = all;
    unsigned long long total = sh.first.weight[(1 << FIRST) - 1];
    auto cut = [&](uint32_t to) {
        const SamplePlace p = place(true, to);
        stay = to;
        total = p.weight_before + (to - p.before) * weight_of(p.key);
    };
    const int k = a.top_k ? a.top_k[row] : 0;
    if (greedy || (k > 0 && (uint32_t)k < all)) cut(greedy ? 1u : (uint32_t)k);
    const float p = a.top_p ? a.top_p[row] : 1.f;
    if (p < 1.f && stay > 1) {
        unsigned long long want = p > 0.f ? sample_share(p, total, true) : 0;
        want = want < 1 ? 1 : want;
        const SamplePlace at = place(false, want);
        const unsigned long long w = weight_of(at.key), some = (want - at.weight_before + w - 1) / w;
        stay = at.before + (uint32_t)some;
        total = at.weight_before + some * w;
    }
    if ((uint32_t)likely < stay) cut((uint32_t)likely);

    float u = a.u[row];
    u = u > 0.f ? (u < 1.f ? u : 0x1.fffffep-1f) : 0.f;
    const unsigned long long want = sample_share(u, total, false) + 1;
    const SamplePlace at = place(false, want);
    const unsigned long long w = weight_of(at.key);
    // the nth of the logits of that value
    uint32_t nth = (uint32_t)((want - at.weight_before + w - 1) / w);
    if (at.n <= (uint32_t)SAMPLE_LIST) {
        __syncthreads();
        each([&](uint32_t x, int i) {
            if (key_of(x) == at.key) sh.list[atomicAdd(&sh.listed, 1)] = i;
        });
        __syncthreads();
        if (t < (int)at.n) {
            const int mine = sh.list[t];
            uint32_t r = 0;
            for (uint32_t j = 0; j < at.n; ++j) r += sh.list[j] < mine ? 1u : 0u;
            if (r + 1 == nth) sh.token = mine;
        }
        __syncthreads();
    } else {
        // by their indices' bits, from the highest
        int prefix = 0;
        for (int down = 33; down > 0;) {
            const int bits = SAMPLE_BITS, next = down - bits;
            __syncthreads();
            sample_clear(sh.next);
            __syncthreads();
            each([&](uint32_t x, int i) {
                if (key_of(x) == at.key && (down > 31 || i >> down == prefix)) atomicAdd(&sh.next.count[(i >> next) & (SAMPLE_BINS - 1)], 1u);
            });
            __syncthreads();
            sample_sums(sh, sh.next);
            const int bin = search(sh.next, true, nth);
            nth -= bin ? sh.next.count[bin - 1] : 0;
            prefix = prefix << bits | bin;
            down = next;
        }
        if (t == 0) sh.token = prefix;
        __syncthreads();
    }
    if (t == 0) {
        a.token[row] = sh.token;
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

}  // namespace pnn

using namespace pnn;

extern "C" size_t posit_sample_workspace(int fz, int64_t rows, int64_t vocab) {
    (void)fz; (void)rows; (void)vocab;
    return 0;
}

extern "C" int posit_sample(void* stream, int fz, int64_t rows, int64_t vocab, const void* logits, int64_t ldz, const float* u, const float* temperature, const int32_t* top_k,
                            const float* top_p, const float* min_p, int32_t* token, float* logprob, int32_t* kept, void* workspace, size_t workspace_bytes) {
    if (rows < 0 || vocab < 0 || ldz < vocab) return PNN_EINVAL;
    if (const int s = element_status(fz)) return s;
    if (vocab >= ((int64_t)1 << 31) || rows >= ((int64_t)1 << 31)) return PNN_EUNSUPPORTED;
    if (rows == 0 || vocab == 0) return PNN_OK;
    if (!logits || !u || !token) return PNN_EINVAL;
    (void)workspace; (void)workspace_bytes;
    hipStream_t st = (hipStream_t)stream;
    discard_stale_hip_error();
    Sample a = {logits, u, temperature, top_p, min_p, top_k, token, kept, logprob, vocab, ldz, sample_shift(vocab), elem_fmt(fz), 0};
    for (const int64_t most = most_workgroups(SAMPLE_THREADS); a.row0 < rows; a.row0 += most) {
        const unsigned n = (unsigned)(rows - a.row0 < most ? rows - a.row0 : most);
        PNN_DISPATCH_KIND(kind_of(fz), hipLaunchKernelGGL(sample_kernel<K>, dim3(n), dim3(SAMPLE_THREADS), 0, st, a))
    }
    return hip_status(hipGetLastError());
}
