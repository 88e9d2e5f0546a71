// The choice of a token from its logits (include/ogc_sample.h).
//
// What is kept is always the beginning of the tokens in the order of falling logits, so that a limit comes down to one logit and how many of the
// tokens that have it are kept, the lowest indices first.  No row is sorted: the limit's logit is found digit by digit of its 32-bit
// key (11, 11 and 10 bits), from the counts and the weights of the tokens with each digit.  Weights are whole numbers of 2^-42: their
// sums have no rounding, so that neither the order in which wavefronts add nor the way in which a row is shared changes a token.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "ogc_sample.h"

#define SAMPLE_DEV static __device__ __forceinline__

namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

struct SampleArgs {
    const uint8_t* logits;
    const float* temperature;  // or NULL, the next three as well
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    const float* uniform;
    int32_t* tokens;
    float* logs;  // or NULL
    long long stride;  // bytes
    int rows, vocab;
};

constexpr int THREADS = 1024, WAVES = THREADS / 64, BINS = 2048;

// A logit as a key that compares the same way; NaN as minus infinity, -0 as 0.
SAMPLE_DEV uint32_t key_of(float x) {
    x = x == x ? x + 0.0f : -INFINITY;
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    return b >> 31 ? ~b : b | 0x80000000u;
}
SAMPLE_DEV float logit_of(uint32_t key) { return __builtin_bit_cast(float, key >> 31 ? key & 0x7fffffffu : ~key); }
constexpr uint32_t NOTHING = 0x007fffffu;  // the key of minus infinity

template <int DT> SAMPLE_DEV float logit_at(const uint8_t* row, int i) {
    if constexpr (DT == OGC_F32) return ((const float*)row)[i];
    else return __builtin_bit_cast(float, (uint32_t)((const uint16_t*)row)[i] << 16);
}

// Weights of a row: multiples of 2^-42, in 64 bits.
struct Weights {
    double largest, per;  // 1 / temperature
    __device__ __forceinline__ double log_of(float logit) const {
        const double x = logit;
        return x == largest ? 0.0 : (x - largest) * per;
    }
    // 2^42 exp(x), rounded.  x / ln 2 = n + f, |f| <= 1/2; the series of exp(f ln 2) ends below 2^-47.
    static __device__ __forceinline__ uint64_t of_log(double x) {
        if (!(x > -29.9)) return 0;  // (below half of 2^-42)
        const double y = x * 1.44269504088896340736;
        const double n = __builtin_rint(y), f = (y - n) * 0.693147180559945309417;
        double p = 1.0 / 39916800;
        p = __builtin_fma(p, f, 1.0 / 3628800);
        p = __builtin_fma(p, f, 1.0 / 362880);
        p = __builtin_fma(p, f, 1.0 / 40320);
        p = __builtin_fma(p, f, 1.0 / 5040);
        p = __builtin_fma(p, f, 1.0 / 720);
        p = __builtin_fma(p, f, 1.0 / 120);
        p = __builtin_fma(p, f, 1.0 / 24);
        p = __builtin_fma(p, f, 1.0 / 6);
        p = __builtin_fma(p, f, 0.5);
        p = __builtin_fma(p, f, 1.0);
        p = __builtin_fma(p, f, 1.0);
        const double v = __builtin_ldexp(p, (int)n + 42);  // at most 2^42
        return __builtin_bit_cast(uint64_t, v + 0x1p52) - 0x4330000000000000ull;
    }
    __device__ __forceinline__ uint64_t of(uint32_t key) const { return key == NOTHING ? 0 : of_log(log_of(logit_of(key))); }
};

struct Shared {
    uint64_t mass[BINS];
    uint32_t count[BINS];
    uint64_t part[2][WAVES];
    uint64_t got[3];
    uint32_t found[2];
};

SAMPLE_DEV uint64_t shfl(uint64_t x, int from) {
    const uint32_t lo = __shfl((uint32_t)x, from), hi = __shfl((uint32_t)(x >> 32), from);
    return (uint64_t)hi << 32 | lo;
}
SAMPLE_DEV uint64_t shfl_up(uint64_t x, int by) {
    const uint32_t lo = __shfl_up((uint32_t)x, by), hi = __shfl_up((uint32_t)(x >> 32), by);
    return (uint64_t)hi << 32 | lo;
}
SAMPLE_DEV uint64_t wave_upto(uint64_t x, int lane) {  // sum over the lanes up to this one
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const uint64_t t = shfl_up(x, m);
        if (lane >= m) x += t;
    }
    return x;
}
SAMPLE_DEV uint64_t wave_sum(uint64_t x, int lane) { return shfl(wave_upto(x, lane), 63); }

// What is kept: the keys above `key`, and the first `ties` of the tokens that have it.
struct Limit {
    uint32_t key;
    uint32_t ties;
    uint64_t mass;  // of all that is kept
};

// The tokens that are kept by `outer` and, of them in falling order, the first `k` (or fewer: there may not be so many), or the fewest whose weights add up to
// a share of all of theirs.
template <int DT> SAMPLE_DEV Limit select(Shared& sh, const uint8_t* row, int vocab, const Weights& weights, const Limit& outer, bool by_mass, uint32_t k, double share) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t prefix = 0;
    uint64_t want = k, before_mass = 0;
    Limit r = outer;
#pragma unroll
    for (int digit = 0; digit < 3; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bins = digit == 2 ? 1024 : 2048;
        __syncthreads();
        for (int i = threadIdx.x; i < BINS; i += THREADS) sh.mass[i] = 0, sh.count[i] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < vocab; i += THREADS) {
            const uint32_t key = key_of(logit_at<DT>(row, i));
            if (key <= outer.key) continue;
            if (digit == 1 && key >> 21 != prefix) continue;
            if (digit == 2 && key >> 10 != prefix) continue;
            const uint64_t w = weights.of(key);
            if (w == 0) continue;
            const int b = key >> shift & (bins - 1);
            atomicAdd((unsigned long long*)&sh.mass[b], (unsigned long long)w);
            atomicAdd(&sh.count[b], 1u);
        }
        __syncthreads();
        if (threadIdx.x == 0 && outer.ties) {  // equal ones: so many of them as are there
            const uint32_t key = outer.key;
            if (digit == 0 || (digit == 1 && key >> 21 == prefix) || (digit == 2 && key >> 10 == prefix)) {
                sh.mass[key >> shift & (bins - 1)] += outer.ties * weights.of(key);
                sh.count[key >> shift & (bins - 1)] += outer.ties;
            }
        }
        __syncthreads();
        // two bins a thread, from the top
        const int hi = bins - 1 - 2 * (int)threadIdx.x;
        const bool mine = hi >= 0;
        const uint64_t m0 = mine ? sh.mass[hi] : 0, m1 = mine ? sh.mass[hi - 1] : 0;
        const uint64_t c0 = mine ? sh.count[hi] : 0, c1 = mine ? sh.count[hi - 1] : 0;
        uint64_t ms = wave_upto(m0 + m1, lane), cs = wave_upto(c0 + c1, lane);
        if (lane == 63) sh.part[0][wave] = ms, sh.part[1][wave] = cs;
        __syncthreads();
        uint64_t all_mass = 0, all_count = 0;
        for (int i = 0; i < WAVES; ++i) {
            if (i < wave) ms += sh.part[0][i], cs += sh.part[1][i];
            all_mass += sh.part[0][i], all_count += sh.part[1][i];
        }
        if (digit == 0) {
            if (by_mass) {
                const double t = __builtin_ceil(share * (double)all_mass);
                want = t >= (double)all_mass ? all_mass : (uint64_t)t;
                if (want == 0) want = 1;
            } else if (want >= all_count) {
                r.mass = all_mass;  // all of them
                return r;
            }
        }
        // the bin in which the wanted amount is reached
        const uint64_t end = by_mass ? ms : cs, x0 = by_mass ? m0 : c0, x1 = by_mass ? m1 : c1, start = end - x0 - x1;
        if (mine && start < want && want <= end) {
            const bool first = want <= start + x0;
            sh.found[0] = first ? hi : hi - 1;
            sh.got[0] = first ? start : start + x0;                                        // of what is counted, before the bin
            sh.got[1] = first ? ms - m0 - m1 : ms - m1;                                    // mass before it
        }
        __syncthreads();
        prefix = digit == 0 ? sh.found[0] : digit == 1 ? prefix << 11 | sh.found[0] : prefix << 10 | sh.found[0];
        want -= sh.got[0];
        before_mass += sh.got[1];
    }
    const uint64_t w = weights.of(prefix);
    r.key = prefix;
    r.ties = by_mass ? (uint32_t)((want + w - 1) / w) : (uint32_t)want;
    r.mass = before_mass + r.ties * w;
    __syncthreads();
    return r;
}

// What of the tokens first .. last - 1 is kept, for a wavefront: the weight of those above the limit, and how many are at it.
template <int DT> SAMPLE_DEV void range_of(const uint8_t* row, int first, int last, const Weights& weights, const Limit& limit, double least, int lane,
                                           uint64_t& mass, uint32_t& ties) {
    uint64_t m = 0, t = 0;
    for (int i = first + lane; i < last; i += 64) {
        const uint32_t key = key_of(logit_at<DT>(row, i));
        if (key == NOTHING) continue;
        t += key == limit.key;
        if (key > limit.key) {
            const double x = weights.log_of(logit_of(key));
            m += x >= least ? Weights::of_log(x) : 0;
        }
    }
    mass = wave_sum(m, lane);
    ties = (uint32_t)wave_sum(t, lane);
}

template <int DT> __global__ __launch_bounds__(THREADS) void ogc_sample_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = blockIdx.x, vocab = a.vocab;
    const uint8_t* const row = a.logits + r * a.stride;

    uint32_t top = NOTHING;
    for (int i = threadIdx.x; i < vocab; i += THREADS) top = max(top, key_of(logit_at<DT>(row, i)));
#pragma unroll
    for (int m = 1; m < 64; m *= 2) top = max(top, (uint32_t)__shfl_xor(top, m));
    if (lane == 0) sh.found[0] = 0, sh.part[0][wave] = top;
    __syncthreads();
    for (int i = 0; i < WAVES; ++i) top = max(top, (uint32_t)sh.part[0][i]);
    __syncthreads();
    if (top == NOTHING) {
        if (threadIdx.x == 0) {
            a.tokens[r] = -1;
            if (a.logs) a.logs[r] = -INFINITY;
        }
        return;
    }
    const float t = a.temperature ? a.temperature[r] : 1.0f;
    const int k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.0f, low = a.min_p ? a.min_p[r] : 0.0f;
    const bool greedy = !(t > 0.0f);
    Weights weights;
    weights.largest = logit_of(top);
    weights.per = greedy ? 0.0 : 1.0 / (double)t;

    Limit limit = {NOTHING, 0, 0};
    if (greedy) limit.key = top, limit.ties = 1;
    else {
        if (k > 0 && k < vocab) limit = select<DT>(sh, row, vocab, weights, limit, false, (uint32_t)k, 0.0);
        if (p < 1.0f) limit = select<DT>(sh, row, vocab, weights, limit, true, 0, p > 0.0f ? (double)p : 0.0);
    }
    const double least = low > 0.0f ? (low < 1.0f ? log((double)low) : 0.0) : -INFINITY;
    const double at_limit = limit.ties ? weights.log_of(logit_of(limit.key)) : 0.0;
    const uint64_t tie = limit.ties && at_limit >= least ? Weights::of_log(at_limit) : 0;

    // The running sum by index, in three steps: a sixteenth of the row for each wavefront, a sixteenth of the one that holds the token, and
    // the tokens of that.
    const int wide = (vocab + WAVES * 64 - 1) / (WAVES * 64) * 64;
    int first = 0, width = wide;
    uint64_t before = 0, target = 0, total = 0;
    uint32_t ties_before = 0;
#pragma unroll
    for (int level = 0; level < 2; ++level) {
        const int b = min(first + wave * width, vocab), e = min(min(b + width, vocab), level == 0 ? vocab : first + wide);
        uint64_t mass;
        uint32_t ties;
        range_of<DT>(row, b, e, weights, limit, least, lane, mass, ties);
        __syncthreads();
        if (lane == 0) sh.part[0][wave] = mass, sh.part[1][wave] = ties;
        __syncthreads();
        uint64_t run = before;
        uint32_t seen = ties_before;
        int found = 0;
        uint64_t found_run = before;
        uint32_t found_seen = ties_before;
        if (level == 0) {
            for (int i = 0; i < WAVES; ++i) {
                const uint32_t n = min((uint32_t)sh.part[1][i], limit.ties - min(limit.ties, seen));
                total += sh.part[0][i] + n * tie;
                seen += (uint32_t)sh.part[1][i];
            }
            seen = 0;
            const float u = a.uniform[r];
            const double at = __builtin_floor((u > 0.0f ? (double)u : 0.0) * (double)total);
            target = at >= (double)total ? total - 1 : (uint64_t)at;
            if (target >= total) target = total - 1;
        }
        for (int i = 0; i < WAVES; ++i) {
            const uint32_t n = min((uint32_t)sh.part[1][i], limit.ties - min(limit.ties, seen));
            const uint64_t here = sh.part[0][i] + n * tie;
            if (run <= target && target < run + here) found = i, found_run = run, found_seen = seen;
            run += here;
            seen += (uint32_t)sh.part[1][i];
        }
        first += found * width;
        before = found_run;
        ties_before = found_seen;
        if (level == 0) width = (width + WAVES * 64 - 1) / (WAVES * 64) * 64;
    }
    if (wave != 0) return;
    const int last = min(min(first + width, vocab), vocab);
    for (int i0 = first; i0 < last; i0 += 64) {
        const int i = i0 + lane;
        const uint32_t key = i < last ? key_of(logit_at<DT>(row, i)) : NOTHING;
        const double x = key == NOTHING ? 0.0 : weights.log_of(logit_of(key));
        const bool equal = key == limit.key && key != NOTHING;
        const uint64_t equals = __ballot(equal);
        const uint32_t rank = ties_before + (uint32_t)__popcll(equals & ((1ull << lane) - 1));
        uint64_t w = 0;
        if (key != NOTHING && x >= least && (key > limit.key || (equal && rank < limit.ties))) w = Weights::of_log(x);
        const uint64_t upto = before + wave_upto(w, lane);
        const uint64_t over = __ballot(upto > target);
        if (over) {
            if (lane == __ffsll((unsigned long long)over) - 1) {
                a.tokens[r] = i;
                if (a.logs) a.logs[r] = greedy ? 0.0f : (float)(x - log((double)total * 0x1p-42));
            }
            return;
        }
        before = shfl(upto, 63);
        ties_before += (uint32_t)__popcll(equals);
    }
}

}  // namespace

extern "C" {

ogc_status ogc_sample_validate(const ogc_sample_desc* d) {
    if (!d) return OGC_ERR_INVALID_ARG;
    if (d->dtype < OGC_F32 || d->dtype > OGC_F8) return OGC_ERR_INVALID_ARG;
    if (d->rows < 0 || d->rows > 65535 || d->vocab <= 0 || d->vocab > 1 << 20 || d->stride < d->vocab) return OGC_ERR_SHAPE;
    if (d->dtype != OGC_F32 && d->dtype != OGC_BF16) return OGC_ERR_UNSUPPORTED;
    return OGC_OK;
}

ogc_status ogc_sample_workspace_bytes(const ogc_sample_desc* d, size_t* bytes) {
    const ogc_status st = ogc_sample_validate(d);
    if (st != OGC_OK) return st;
    if (!bytes) return OGC_ERR_INVALID_ARG;
    *bytes = 0;
    return OGC_OK;
}

ogc_status ogc_sample_run(const ogc_sample_desc* d, const void* logits, const float* temperature, const int32_t* top_k,
                          const float* top_p, const float* min_p, const float* uniform, int32_t* tokens, float* log_probabilities,
                          void* workspace, void* stream) {
    const ogc_status st = ogc_sample_validate(d);
    if (st != OGC_OK) return st;
    if (d->rows == 0) return OGC_OK;
    if (!logits || !uniform || !tokens) return OGC_ERR_INVALID_ARG;
    if ((uintptr_t)logits & (d->dtype == OGC_F32 ? 3 : 1)) return OGC_ERR_ALIGNMENT;
    if (((uintptr_t)temperature | (uintptr_t)top_k | (uintptr_t)top_p | (uintptr_t)min_p | (uintptr_t)uniform | (uintptr_t)tokens | (uintptr_t)log_probabilities) & 3)
        return OGC_ERR_ALIGNMENT;
    (void)workspace;
    SampleArgs a;
    a.logits = (const uint8_t*)logits;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.uniform = uniform;
    a.tokens = tokens;
    a.logs = log_probabilities;
    a.stride = d->stride * (d->dtype == OGC_F32 ? 4 : 2);
    a.rows = d->rows;
    a.vocab = d->vocab;
    const hipStream_t s = (hipStream_t)stream;
    if (d->dtype == OGC_F32) hipLaunchKernelGGL((ogc_sample_kernel<OGC_F32>), dim3(d->rows), dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL((ogc_sample_kernel<OGC_BF16>), dim3(d->rows), dim3(THREADS), 0, s, a);
    return hipGetLastError() == hipSuccess ? OGC_OK : OGC_ERR_DEVICE;
}

}  // extern "C"
