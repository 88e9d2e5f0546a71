// The choice of a token from its logits (include/ogc_sample.h).
//
// What is kept is always the beginning of the tokens in the order of falling logits, so that all limits come down to one token, the last kept
// one.  No row is sorted.  A first kernel reads the rows once, in parts, and leaves what a row's choice needs of them: the largest of every eight
// logits, of every part the largest and, with it for the unit, the sum of its weights, or their sums in bins of 1/32 of a temperature.  A second one has
// a workgroup for each row:
//     top-k       at least k of the largest-of-eight are the k-th of them or larger: the tokens that are as large are sorted, a few more than k
//     top-p, min-p  the bins say in which of them the last kept token is: its tokens are sorted
//     the choice    by the kept weight of the parts, then the tokens of one part (top-k: the kept ones, sorted by index)
// Weights are 64-bit values or whole multiples of 2^-42; sums are of whole numbers or in a fixed order, so that a call gives the same tokens every time.
// What that does not cover (more than 1024 for top-k, thousands of equal logits at the limit, logits of plus infinity or 2^17 temperatures)
// takes the row as a whole: the limit's logit digit by digit of its 32-bit key (11, 11 and 10 bits), from the counts and the weights of the tokens with
// each digit.
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
    int parts, chunks;  // of a row: parts of `part` tokens, chunks of eight
    int part;
    int even;           // rows are 16-byte aligned
    float* largest;     // [rows][parts]
    uint64_t* mass;     // [rows][parts]
    float* tops;        // [rows][chunks]
    uint64_t* bins;     // [rows][parts][FINE]
};

constexpr int THREADS = 1024, WAVES = THREADS / 64, BINS = 2048;
constexpr int SCAN_THREADS = 256, FINE = 1024, MOST_K = 1024, MOST = 4096, MOST_PARTS = 256;  // bins of a part; tokens that are sorted

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

struct WholeRow {
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
template <int DT> SAMPLE_DEV Limit select(WholeRow& sh, const uint8_t* row, int vocab, const Weights& weights, const Limit& outer, bool by_mass, uint32_t k, double share) {
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

// A row's limits.
struct Limits {
    bool greedy, top_k, top_p, min_p;
    int k;
    double p, least, per;  // least: the smallest log of a kept weight; per: 1 / temperature
    float fine;            // bins of a logit
};
SAMPLE_DEV Limits limits_of(const SampleArgs& a, int r) {
    const float t = a.temperature ? a.temperature[r] : 1.0f, p = a.top_p ? a.top_p[r] : 1.0f, low = a.min_p ? a.min_p[r] : 0.0f;
    Limits l;
    l.k = a.top_k ? a.top_k[r] : 0;
    l.greedy = !(t > 0.0f);
    l.top_k = l.k > 0 && l.k < a.vocab;
    l.top_p = p < 1.0f;
    l.min_p = low > 0.0f;
    l.p = p > 0.0f ? (double)p : 0.0;
    l.least = l.min_p ? (low < 1.0f ? log((double)low) : 0.0) : -INFINITY;
    l.per = l.greedy ? 0.0 : 1.0 / (double)t;
    l.fine = (float)(32.0 * l.per);
    return l;
}
// A row's choice by the bins of its parts' weights: neither by its largest logits alone (top-k) nor without limits.
SAMPLE_DEV bool by_bins(const Limits& l) { return !l.greedy && !l.top_k && (l.top_p || l.min_p); }
// Where a logit is in units of 1/32 of the temperature, as a whole number; the same instructions wherever it is asked for.
SAMPLE_DEV float place_of(float x, float fine) { return __builtin_floorf(x * fine); }

// Eight neighbouring logits; NaN and what is behind the row as minus infinity.
template <int DT> SAMPLE_DEV void eight_of(const uint8_t* row, int i, int vocab, bool even, float (&x)[8]) {
    if (even && i + 8 <= vocab) {
        if constexpr (DT == OGC_F32) {
            const v4u u = *(const v4u*)(row + (int64_t)i * 4), v = *(const v4u*)(row + (int64_t)i * 4 + 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = __builtin_bit_cast(float, (uint32_t)u[e]), x[4 + e] = __builtin_bit_cast(float, (uint32_t)v[e]);
        } else {
            const v4u u = *(const v4u*)(row + (int64_t)i * 2);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __builtin_bit_cast(float, e & 1 ? (uint32_t)u[e / 2] & 0xffff0000u : (uint32_t)u[e / 2] << 16);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = i + e < vocab ? logit_at<DT>(row, i + e) : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = x[e] == x[e] ? x[e] : -INFINITY;
}

// ---- the parts of the rows.  Bound by reading them once, and by an exponential in 64 bits for each logit of the rows whose weights are all added up.
template <int DT, int RUNS> __global__ __launch_bounds__(SCAN_THREADS) void ogc_sample_scan_kernel(SampleArgs a) {
    __shared__ uint64_t bins[FINE];
    __shared__ float most[SCAN_THREADS / 64];
    __shared__ uint64_t sums[SCAN_THREADS / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = blockIdx.y, part = blockIdx.x;
    const uint8_t* const row = a.logits + r * a.stride;
    const Limits l = limits_of(a, r);
    const bool fill = by_bins(l), add = !l.greedy && !l.top_k;
    float x[RUNS][8], top = -INFINITY;
    const int first = part * a.part + threadIdx.x * 8;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) eight_of<DT>(row, first + i * SCAN_THREADS * 8, a.vocab, a.even, x[i]);
    if (fill)
        for (int i = threadIdx.x; i < FINE; i += SCAN_THREADS) bins[i] = 0;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
        float m = x[i][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) m = fmaxf(m, x[i][e]);
        const int at = first + i * SCAN_THREADS * 8;
        if (at < a.vocab) a.tops[(int64_t)r * a.chunks + at / 8] = m;
        top = fmaxf(top, m);
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    if (lane == 0) most[wave] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SCAN_THREADS / 64; ++i) top = fmaxf(top, most[i]);
    const int64_t at = (int64_t)r * a.parts + part;
    if (threadIdx.x == 0) a.largest[at] = top;
    if (!add || top == -INFINITY) {
        if (threadIdx.x == 0) a.mass[at] = 0;
        return;  // (bins of a part without tokens are not looked at)
    }
    Weights weights;
    weights.largest = top;
    weights.per = l.per;
    const float high = place_of(top, l.fine);
    uint64_t sum = 0;
#pragma unroll
    for (int i = 0; i < RUNS; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (x[i][e] == -INFINITY) continue;
            const uint64_t w = Weights::of_log(weights.log_of(x[i][e]));
            sum += w;
            if (fill && w) {
                const float d = high - place_of(x[i][e], l.fine);
                if (d >= 0.0f && d < (float)FINE) atomicAdd((unsigned long long*)&bins[(int)d], (unsigned long long)w);
            }
        }
    sum = wave_sum(sum, lane);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < SCAN_THREADS / 64; ++i) sum += sums[i];
        a.mass[at] = sum;
    }
    if (fill)
        for (int i = threadIdx.x; i < FINE; i += SCAN_THREADS) a.bins[at * FINE + i] = bins[i];
}

struct Chosen {
    uint64_t tokens[MOST];   // key, then the index's complement: falling, the lowest index first
    uint32_t counts[FINE];
    uint64_t kept[MOST_PARTS];
    uint64_t part[WAVES];
    uint32_t count, low;
    int found;
    uint64_t before;
};
union RowShared {
    WholeRow whole;
    Chosen chosen;
};

// sum of x over the threads before this one; `all`: over all threads
SAMPLE_DEV uint64_t sum_before(uint64_t x, uint64_t* part, uint64_t& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t s = wave_upto(x, lane);
    __syncthreads();
    if (lane == 63) part[wave] = s;
    __syncthreads();
    uint64_t base = 0;
    all = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        if (i < wave) base += part[i];
        all += part[i];
    }
    return base + s - x;
}
// Sorts n tokens, falling; n a power of two from 64 on.  Neighbouring pairs up to 64 apart are one wavefront's.
SAMPLE_DEV void sort(uint64_t* v, int n) {
    for (int k = 2; k <= n; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            if (j >= 64) __syncthreads();
            for (int t = threadIdx.x; t < n / 2; t += THREADS) {
                const int i = 2 * t - (t & (j - 1));
                const uint64_t x = v[i], y = v[i + j];
                if ((x < y) == ((i & k) == 0)) v[i] = y, v[i + j] = x;
            }
            if (j >= 64) __syncthreads();
            else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    __syncthreads();
}
SAMPLE_DEV int padded(uint64_t* v, int n) {  // zeros behind the tokens, which sort last
    int to = 64;
    while (to < n) to *= 2;
    for (int i = n + threadIdx.x; i < to; i += THREADS) v[i] = 0;
    __syncthreads();
    return to;
}
SAMPLE_DEV uint32_t key_in(uint64_t token) { return (uint32_t)(token >> 32); }
SAMPLE_DEV int index_in(uint64_t token) { return (int)~(uint32_t)token; }

// The row as a whole, from its logits alone.
template <int DT> SAMPLE_DEV void whole_row(const SampleArgs& a, WholeRow& sh, const uint8_t* row, const Limits& l, const Weights& weights) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = blockIdx.x, vocab = a.vocab;
    Limit limit = {NOTHING, 0, 0};
    if (l.top_k) limit = select<DT>(sh, row, vocab, weights, limit, false, (uint32_t)l.k, 0.0);
    if (l.top_p) limit = select<DT>(sh, row, vocab, weights, limit, true, 0, l.p);
    const double least = l.least;
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
                if (a.logs) a.logs[r] = (float)(x - log((double)total * 0x1p-42));
            }
            return;
        }
        before = shfl(upto, 63);
        ties_before += (uint32_t)__popcll(equals);
    }
}

// Collects the tokens of the chunks whose largest logit passes `chunk` and that pass `token` themselves; fail is set where there are more than MOST.
template <int DT, class C, class T> SAMPLE_DEV void collect(const SampleArgs& a, Chosen& sh, const uint8_t* row, C chunk, T token) {
    const float* const tops = a.tops + (int64_t)blockIdx.x * a.chunks;
    for (int i0 = 0; i0 < a.chunks; i0 += 4 * THREADS) {
        float m[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + u * THREADS + threadIdx.x;
            m[u] = i < a.chunks ? tops[i] : -INFINITY;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + u * THREADS + threadIdx.x;
            if (m[u] == -INFINITY || !chunk(m[u])) continue;
            float x[8];
            eight_of<DT>(row, i * 8, a.vocab, a.even, x);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (x[e] != -INFINITY && token(x[e])) {
                    const uint32_t to = atomicAdd(&sh.count, 1u);
                    if (to < MOST) sh.tokens[to] = (uint64_t)key_of(x[e]) << 32 | (uint32_t)~(uint32_t)(i * 8 + e);
                }
        }
    }
    __syncthreads();
}

// The running sum that the chosen token's exceeds.
SAMPLE_DEV uint64_t target_of(float u, uint64_t all) {
    const double t = __builtin_floor((u > 0.0f ? (double)u : 0.0) * (double)all);
    return t < (double)all && (uint64_t)t < all ? (uint64_t)t : all - 1;
}
// The weight that the kept tokens add up to, or more.
SAMPLE_DEV uint64_t goal_of(double p, uint64_t all) {
    const double t = __builtin_ceil(p * (double)all);
    const uint64_t goal = t < (double)all ? (uint64_t)t : all;
    return goal ? goal : 1;
}
SAMPLE_DEV void give(const SampleArgs& a, int r, int token, double log_weight, uint64_t all) {
    a.tokens[r] = token;
    if (a.logs) a.logs[r] = (float)(log_weight - log((double)all * 0x1p-42));
}

// The choice among `n` tokens, which become sorted by index.  Up to four of them a thread.
SAMPLE_DEV void choose(const SampleArgs& a, Chosen& sh, int n, const Weights& weights, float u, int r) {
    for (int i = threadIdx.x; i < n; i += THREADS) {  // the index's complement first: falling is the lowest index first
        const uint64_t t = sh.tokens[i];
        sh.tokens[i] = t << 32 | t >> 32;
    }
    __syncthreads();
    sort(sh.tokens, padded(sh.tokens, n));
    uint64_t w[4], own = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int i = threadIdx.x * 4 + e;
        w[e] = i < n ? weights.of((uint32_t)sh.tokens[i]) : 0;
        own += w[e];
    }
    uint64_t all, run = sum_before(own, sh.part, all);
    const uint64_t target = target_of(u, all);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (run <= target && target < run + w[e]) {
            const uint64_t t = sh.tokens[threadIdx.x * 4 + e];
            give(a, r, (int)~(uint32_t)(t >> 32), weights.log_of(logit_of((uint32_t)t)), all);
        }
        run += w[e];
    }
}

// How many of the first n sorted tokens are kept by top-p and min-p; `before`: the weight ahead of them.
SAMPLE_DEV int kept_of(Chosen& sh, int n, const Weights& weights, const Limits& l, uint64_t before, uint64_t goal) {
    if (threadIdx.x == 0) sh.found = n;
    uint64_t w[4], own = 0;
    double x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int i = threadIdx.x * 4 + e;
        x[e] = i < n ? weights.log_of(logit_of(key_in(sh.tokens[i]))) : 0.0;
        w[e] = i < n ? Weights::of_log(x[e]) : 0;
        own += w[e];
    }
    uint64_t all, run = before + sum_before(own, sh.part, all);
    int mine = n;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int i = threadIdx.x * 4 + e;
        if (i < mine && (w[e] == 0 || (l.top_p && run >= goal) || !(x[e] >= l.least))) mine = i;
        run += w[e];
    }
    if (mine < n) atomicMin(&sh.found, mine);
    __syncthreads();
    return sh.found;
}

template <int DT> __global__ __launch_bounds__(THREADS) void ogc_sample_kernel(SampleArgs a) {
    __shared__ RowShared shared;
    Chosen& sh = shared.chosen;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = blockIdx.x;
    const uint8_t* const row = a.logits + r * a.stride;
    const float* const largest = a.largest + (int64_t)r * a.parts;
    const uint64_t* const mass = a.mass + (int64_t)r * a.parts;
    const float* const tops = a.tops + (int64_t)r * a.chunks;
    const Limits l = limits_of(a, r);
    const float u = a.uniform[r];
    float top = -INFINITY;
    for (int i = lane; i < a.parts; i += 64) top = fmaxf(top, largest[i]);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    if (top == -INFINITY) {
        if (threadIdx.x == 0) {
            a.tokens[r] = -1;
            if (a.logs) a.logs[r] = -INFINITY;
        }
        return;
    }
    if (l.greedy) {
        if (threadIdx.x == 0) sh.found = 0x7fffffff;
        __syncthreads();
        for (int i = threadIdx.x; i < a.chunks; i += THREADS)
            if (tops[i] == top) {
                atomicMin(&sh.found, i);
                break;
            }
        __syncthreads();
        if (threadIdx.x == 0) {
            float x[8];
            eight_of<DT>(row, sh.found * 8, a.vocab, a.even, x);
            int e = 0;
            while (x[e] != top && e < 7) ++e;
            a.tokens[r] = sh.found * 8 + e;
            if (a.logs) a.logs[r] = 0.0f;
        }
        return;
    }
    Weights weights;
    weights.largest = top;
    weights.per = l.per;
    const float high = place_of(top, l.fine);
    const auto away = [&](float x) { return high - place_of(x, l.fine); };
    const bool limited = l.top_k || l.top_p || l.min_p;
    // places are whole numbers, and near enough to where the logits are, up to 2^22
    if (limited && (!(__builtin_fabsf(high) < 0x1p22f) || (l.top_k && l.k > MOST_K))) return whole_row<DT>(a, shared.whole, row, l, weights);

    if (l.top_k) {
        // ---- the bin of the k-th of the largest-of-eight
        sh.counts[threadIdx.x] = 0;
        if (threadIdx.x == 0) sh.count = 0, sh.low = 0xffffffffu, sh.found = FINE;
        __syncthreads();
        for (int i = threadIdx.x; i < a.chunks; i += THREADS) {
            const float d = away(tops[i]);
            if (d < (float)FINE) atomicAdd(&sh.counts[(int)d], 1u);
        }
        __syncthreads();
        uint64_t all;
        const uint64_t c = sh.counts[threadIdx.x], s = sum_before(c, sh.part, all), k = (uint64_t)l.k;
        if (s < k && k <= s + c) sh.found = threadIdx.x;
        __syncthreads();
        const float bin = (float)sh.found;
        // the smallest of those up to that bin: k tokens at least are as large.  (Fewer than k with a weight: all of them.)
        if (sh.found < FINE) {
            uint32_t low = 0xffffffffu;
            for (int i = threadIdx.x; i < a.chunks; i += THREADS)
                if (away(tops[i]) <= bin) low = min(low, key_of(tops[i]));
            if (low != 0xffffffffu) atomicMin(&sh.low, low);
            __syncthreads();
            const float least = logit_of(sh.low);
            collect<DT>(a, sh, row, [&](float m) { return m >= least; }, [&](float x) { return x >= least; });
        } else {
            collect<DT>(a, sh, row, [&](float m) { return away(m) < (float)FINE; }, [&](float x) { return away(x) < (float)FINE; });
        }
        int n = (int)sh.count;
        __syncthreads();
        if (n > MOST) return whole_row<DT>(a, shared.whole, row, l, weights);
        sort(sh.tokens, padded(sh.tokens, n));
        n = min(n, l.k);
        if (l.top_p || l.min_p) {
            uint64_t own = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) own += threadIdx.x * 4 + e < n ? weights.of(key_in(sh.tokens[threadIdx.x * 4 + e])) : 0;
            sum_before(own, sh.part, all);
            n = kept_of(sh, n, weights, l, 0, goal_of(l.p, all));
        }
        return choose(a, sh, n, weights, u, r);
    }

    // ---- without top-k: the parts' weights in the row's unit
    const auto factor = [&](int p) {
        const double f = largest[p] == top ? 1.0 : exp(((double)largest[p] - (double)top) * l.per);
        return f > 0.0 ? f : 0.0;
    };
    const auto in_row = [&](uint64_t mass, int p) { return (uint64_t)((double)mass * factor(p)); };
    int from = FINE, kept = 0;  // kept: all of the bins before `from`, and the first `kept` sorted tokens
    if (limited) {
        // ---- bins of the row, a thread each
        uint64_t b = 0;
        for (int p = 0; p < a.parts; ++p) {
            const float off = high - place_of(largest[p], l.fine);
            if (largest[p] == -INFINITY || !(off < (float)FINE)) continue;
            const int i = (int)threadIdx.x - (int)off;
            if (i >= 0) b += in_row(a.bins[((int64_t)r * a.parts + p) * FINE + i], p);
        }
        if (threadIdx.x == 0) sh.count = 0, sh.found = FINE - 1;
        uint64_t all;
        const uint64_t s = sum_before(b, sh.part, all), goal = goal_of(l.p, all);
        if (l.top_p && s < goal && goal <= s + b) sh.found = threadIdx.x;
        __syncthreads();
        from = sh.found;
        int to = from;  // the bins that the last kept token may be in
        if (l.min_p) {  // (the threshold's, and the ones beside it: places are rounded down)
            const double x = __builtin_floor(-l.least * 32.0);
            const int near = x < (double)FINE ? (int)x : FINE;
            if (!l.top_p || from >= near - 1) {
                to = min(from, near + 2);
                from = min(max(near - 1, 0), to);
            }
        }
        if ((int)threadIdx.x == from) sh.before = s;
        __syncthreads();
        const uint64_t before = sh.before;
        const float f = (float)from, t = (float)to;
        collect<DT>(a, sh, row, [&](float m) { return away(m) <= t; }, [&](float x) { const float d = away(x); return d >= f && d <= t; });
        const int n = (int)sh.count;
        __syncthreads();
        if (n > MOST) return whole_row<DT>(a, shared.whole, row, l, weights);
        sort(sh.tokens, padded(sh.tokens, n));
        kept = kept_of(sh, n, weights, l, before, goal);
    }
    // ---- the part that has the token: what is kept of each
    const uint64_t end = kept ? sh.tokens[kept - 1] : ~0ull;  // the last of the sorted tokens that are kept
    if (threadIdx.x < MOST_PARTS) sh.kept[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < kept; i += THREADS)
        atomicAdd((unsigned long long*)&sh.kept[index_in(sh.tokens[i]) / a.part], (unsigned long long)weights.of(key_in(sh.tokens[i])));
    if (limited) {
        for (int p = wave; p < a.parts; p += WAVES) {
            const float off = high - place_of(largest[p], l.fine);
            if (largest[p] == -INFINITY || !(off < (float)from)) continue;
            uint64_t m = 0;
            for (int i = lane; i < from - (int)off; i += 64) m += a.bins[((int64_t)r * a.parts + p) * FINE + i];
            m = wave_sum(m, lane);
            if (lane == 0) atomicAdd((unsigned long long*)&sh.kept[p], (unsigned long long)in_row(m, p));
        }
    } else if (threadIdx.x < a.parts) {
        sh.kept[threadIdx.x] = in_row(mass[threadIdx.x], threadIdx.x);
    }
    if (threadIdx.x == 0) sh.found = 0;
    __syncthreads();
    const uint64_t own = threadIdx.x < a.parts ? sh.kept[threadIdx.x] : 0;
    uint64_t total, run = sum_before(own, sh.part, total);
    const uint64_t target = target_of(u, total);
    if (run <= target && target < run + own) sh.found = threadIdx.x, sh.before = run;
    __syncthreads();
    // ---- its tokens, in the part's own unit
    const int p = sh.found;
    const double f = factor(p), rest = (double)(target - sh.before) / f;
    Weights near = weights;
    near.largest = largest[p];
    const int at = p * a.part + (int)threadIdx.x * 8;
    uint64_t w[8], mine = 0;
    float x[8];
    const bool here = (int)threadIdx.x * 8 < a.part && at < a.vocab;
    if (here) eight_of<DT>(row, at, a.vocab, a.even, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        w[e] = 0;
        if (!here || x[e] == -INFINITY) continue;
        const uint64_t token = (uint64_t)key_of(x[e]) << 32 | (uint32_t)~(uint32_t)(at + e);
        if (!limited || away(x[e]) < (float)from || token >= end) w[e] = Weights::of_log(near.log_of(x[e]));
        mine += w[e];
    }
    uint64_t all;
    run = sum_before(mine, sh.part, all);
    const uint64_t goal = rest < (double)all && (uint64_t)rest < all ? (uint64_t)rest : all - 1;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (run <= goal && goal < run + w[e]) give(a, r, at + e, weights.log_of(x[e]), total);
        run += w[e];
    }
}

// Tokens of a part: as many as leave the chip enough workgroups, 8192 at most; 256 parts of a row at most.
int part_of(const ogc_sample_desc* d) {
    int part = 8192;
    while (part > 2048 && (int64_t)d->rows * ((d->vocab + part - 1) / part) < 512 && (d->vocab + part / 2 - 1) / (part / 2) <= MOST_PARTS) part /= 2;
    return part;
}

template <int DT> void launch(const SampleArgs& a, hipStream_t s) {
    const dim3 grid(a.parts, a.rows), threads(SCAN_THREADS);
    if (a.part == 2048) hipLaunchKernelGGL((ogc_sample_scan_kernel<DT, 1>), grid, threads, 0, s, a);
    else if (a.part == 4096) hipLaunchKernelGGL((ogc_sample_scan_kernel<DT, 2>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((ogc_sample_scan_kernel<DT, 4>), grid, threads, 0, s, a);
    hipLaunchKernelGGL((ogc_sample_kernel<DT>), dim3(a.rows), dim3(THREADS), 0, s, a);
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
    const size_t part = (size_t)part_of(d), parts = (d->vocab + part - 1) / part, chunks = (d->vocab + 7) / 8;
    *bytes = d->rows * (parts * (FINE * sizeof(uint64_t) + sizeof(uint64_t) + sizeof(float)) + chunks * sizeof(float));
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
    if (!workspace) return OGC_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15) return OGC_ERR_ALIGNMENT;
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
    a.part = part_of(d);
    a.parts = (d->vocab + a.part - 1) / a.part;
    a.chunks = (d->vocab + 7) / 8;
    a.even = ((uintptr_t)logits | (uintptr_t)a.stride) % 16 == 0;
    a.bins = (uint64_t*)workspace;
    a.mass = a.bins + (size_t)d->rows * a.parts * FINE;
    a.largest = (float*)(a.mass + (size_t)d->rows * a.parts);
    a.tops = a.largest + (size_t)d->rows * a.parts;
    const hipStream_t s = (hipStream_t)stream;
    if (d->dtype == OGC_F32) launch<OGC_F32>(a, s);
    else launch<OGC_BF16>(a, s);
    return hipGetLastError() == hipSuccess ? OGC_OK : OGC_ERR_DEVICE;
}

}  // extern "C"
