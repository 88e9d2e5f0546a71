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
    float* largest;     // [rows][parts]
    uint64_t* mass;     // [rows][parts]
    float* tops;        // [rows][chunks]
    double* bins;       // [rows][parts][FINE]
};

constexpr int THREADS = 1024, WAVES = THREADS / 64, BINS = 2048;
static_assert(WAVES == 16, "the wavefronts' sums are a row of 16 lanes");
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

// Weights of a row (or of a part of it, whose largest logit is then the unit): multiples of 2^-42, in 64 bits.
struct Weights {
    double largest, per;  // 1 / temperature
    __device__ __forceinline__ double log_of(float logit) const {
        const double x = logit;
        return x == largest ? 0.0 : (x - largest) * per;
    }
    // p f + c, with c in scalar registers: written as an expression it costs a copy of c into vector registers each time, a third of all instructions
    static __device__ __forceinline__ double next(double p, double f, double c) {
        asm("v_fma_f64 %0, %0, %1, %2" : "+v"(p) : "v"(f), "s"(c));
        return p;
    }
    // 2^42 2^y, rounded, for y <= 0.  y = n + f, |f| <= 1/2: added to 3 * 2^51, y leaves n in the lower word; 2^f by the polynomial of degree 9 through its
    // values at the ten Chebyshev points, off by 2^-45.6; n goes into its exponent; and added to 2^52, what is left of the point is in the lower 52 bits.
    static __device__ __forceinline__ uint64_t of_log2(double y) {
        y = __builtin_fmax(y, -64.0);  // (no weight from -43 on)
        const double t = y + 0x1.8p52, f = y - (t - 0x1.8p52);
        double p = 0x1.b6571de2f2351p-24;
        p = next(p, f, 0x1.63ef969a64d3cp-20);
        p = next(p, f, 0x1.ffcb76789860fp-17);
        p = next(p, f, 0x1.43088e257f341p-13);
        p = next(p, f, 0x1.5d87fe908f88ap-10);
        p = next(p, f, 0x1.3b2ab72b175eep-7);
        p = next(p, f, 0x1.c6b08d7044119p-5);
        p = next(p, f, 0x1.ebfbdff8149f2p-3);
        p = next(p, f, 0x1.62e42fefa39f7p-1);
        p = next(p, f, 0x1.000000000003dp+0);
        const uint64_t bits = __builtin_bit_cast(uint64_t, p) + ((uint64_t)(((uint32_t)__builtin_bit_cast(uint64_t, t) + 42) << 20) << 32);
        return __builtin_bit_cast(uint64_t, __builtin_bit_cast(double, bits) + 0x1p52) & 0xfffffffffffffull;
    }
    static __device__ __forceinline__ uint64_t of_log(double x) { return of_log2(x * 1.44269504088896340736); }
    // of a logit, which is at most the largest (or NaN: none), where that is finite: the same instructions wherever a part's weights are added up
    __device__ __forceinline__ uint64_t of_part(float logit) const { return of_log2(((double)logit - largest) * (per * 1.44269504088896340736)); }
    // where it is plus infinity
    static __device__ __forceinline__ uint64_t of_infinite(float logit) { return logit == INFINITY ? 1ull << 42 : 0; }
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
// x of another lane of the wavefront, 0 where there is none
template <int CTRL, int ROWS> SAMPLE_DEV uint64_t moved(uint64_t x) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xf, false);
    return (uint64_t)hi << 32 | lo;
}
SAMPLE_DEV uint64_t row_upto(uint64_t x) {  // sum over the lanes of 16 up to this one
    x += moved<0x111, 0xf>(x);  // 1, 2, 4, 8 lanes before
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    return x + moved<0x118, 0xf>(x);
}
SAMPLE_DEV uint64_t wave_upto(uint64_t x) {  // sum over the lanes up to this one
    x = row_upto(x);
    x += moved<0x142, 0xa>(x);  // the last lane of the 16 before, for the second and the fourth 16
    return x + moved<0x143, 0xc>(x);  // lane 31, for the upper half
}
SAMPLE_DEV uint64_t lane_of(uint64_t x, int lane) {  // the same lane for all
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)x, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane);
    return (uint64_t)hi << 32 | lo;
}
SAMPLE_DEV uint64_t wave_sum(uint64_t x) { return lane_of(wave_upto(x), 63); }

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
#pragma unroll 1
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
        uint64_t ms = wave_upto(m0 + m1), cs = wave_upto(c0 + c1);
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
    mass = wave_sum(m);
    ties = (uint32_t)wave_sum(t);
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

// A row's chunks are the eights of its memory, not of its indices: chunk c begins with token 8 c - off, where off of the row's first bytes are missing
// to a multiple of 16.  All chunks but the first and the last are then loaded whole, whatever the rows' stride.
template <int DT> SAMPLE_DEV int off_of(const uint8_t* row) { return (int)((uintptr_t)row & 15) / (DT == OGC_F32 ? 4 : 2); }
// Eight neighbouring logits from token i on (a chunk's first, perhaps before the row); what is not the row's is minus infinity.
template <int DT> struct Eight {
    v4u raw[DT == OGC_F32 ? 2 : 1];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < (DT == OGC_F32 ? 2 : 1); ++i) {
            const uint32_t none = DT == OGC_F32 ? 0xff800000u : 0xff80ff80u;
            raw[i] = (v4u){none, none, none, none};
        }
    }
    __device__ __forceinline__ void load(const uint8_t* row, int i, int vocab) {
        if (i >= 0 && i + 8 <= vocab) whole(row, i);
        else part(row, i, vocab);
    }
    __device__ __forceinline__ void whole(const uint8_t* row, int i) {
        const uint8_t* const p = row + (int64_t)i * (DT == OGC_F32 ? 4 : 2);
        raw[0] = *(const v4u*)p;
        if constexpr (DT == OGC_F32) raw[1] = *(const v4u*)(p + 16);
    }
    __device__ __forceinline__ void part(const uint8_t* row, int i, int vocab) {
        clear();
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {  // (a row has two such chunks at most: short code is worth more than their time)
            next();
            if (i + e < 0 || i + e >= vocab) continue;
            if constexpr (DT == OGC_F32) raw[1][3] = ((const uint32_t*)row)[i + e];
            else raw[0][3] = (raw[0][3] & 0xffffu) | (uint32_t)((const uint16_t*)row)[i + e] << 16;
        }
    }
    __device__ __forceinline__ void next() {  // logit 1 in the place of logit 0, and so on
        if constexpr (DT == OGC_F32) {
            const uint32_t first = raw[0][0];
            raw[0] = (v4u){raw[0][1], raw[0][2], raw[0][3], raw[1][0]};
            raw[1] = (v4u){raw[1][1], raw[1][2], raw[1][3], first};
        } else {
            const v4u t = raw[0];
            raw[0] = (v4u){t[0] >> 16 | t[1] << 16, t[1] >> 16 | t[2] << 16, t[2] >> 16 | t[3] << 16, t[3] >> 16 | t[0] << 16};
        }
    }
    __device__ __forceinline__ float get(int e) const {  // (NaN as it is)
        if constexpr (DT == OGC_F32) return __builtin_bit_cast(float, (uint32_t)raw[e / 4][e % 4]);
        else return __builtin_bit_cast(float, e & 1 ? (uint32_t)raw[0][e / 2] & 0xffff0000u : (uint32_t)raw[0][e / 2] << 16);
    }
    __device__ __forceinline__ float number(int e) const {  // NaN as minus infinity
        const float x = get(e);
        return x == x ? x : -INFINITY;
    }
};

// ---- the parts of the rows.  Bound by reading them once (64 rows of 128000 fp32 logits 6.6 us, 5.0 TB/s), and by an exponential in 64 bits for each logit of the
// rows whose weights are all added up (14.3 us; with bins 18.2).
template <int DT, int RUNS> __global__ __launch_bounds__(SCAN_THREADS) void ogc_sample_scan_kernel(SampleArgs a) {
    __shared__ uint64_t bins[FINE];
    __shared__ float most[SCAN_THREADS / 64];
    __shared__ uint64_t sums[SCAN_THREADS / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = blockIdx.y, part = blockIdx.x;
    const uint8_t* const row = a.logits + r * a.stride;
    const Limits l = limits_of(a, r);
    const bool fill = by_bins(l), add = !l.greedy && !l.top_k;
    Eight<DT> x[RUNS];
    float top = -INFINITY;
    const int off = off_of<DT>(row), first = part * a.part + threadIdx.x * 8;  // (of the chunks)
#pragma unroll
    for (int i = 0; i < RUNS; ++i) x[i].load(row, first + i * SCAN_THREADS * 8 - off, a.vocab);
    if (fill)
        for (int i = threadIdx.x; i < FINE; i += SCAN_THREADS) bins[i] = 0;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
        float m = x[i].number(0);
#pragma unroll
        for (int e = 1; e < 8; ++e) m = fmaxf(m, x[i].number(e));
        const int at = (first + i * SCAN_THREADS * 8) / 8;
        if (at < a.chunks) a.tops[(int64_t)r * a.chunks + at] = m;
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
    const bool infinite = __builtin_amdgcn_readfirstlane(top == INFINITY);
    uint64_t sum = 0;
#pragma unroll 1
    for (int i = 0; i < RUNS; ++i) {  // (one after the other through x[0]: eight exponentials side by side keep the pipe busy)
        uint64_t w[8];
        if (infinite) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = Weights::of_infinite(x[0].get(e));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = weights.of_part(x[0].get(e));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += w[e];
        if (fill) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = high - place_of(x[0].get(e), l.fine);
                if (w[e] && d >= 0.0f && d < (float)FINE) atomicAdd((unsigned long long*)&bins[(int)d], (unsigned long long)w[e]);
            }
        }
#pragma unroll
        for (int j = 0; j + 1 < RUNS; ++j) x[j] = x[j + 1];
    }
    sum = wave_sum(sum);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < SCAN_THREADS / 64; ++i) sum += sums[i];
        a.mass[at] = sum;
    }
    if (fill)
        for (int i = threadIdx.x; i < FINE; i += SCAN_THREADS) a.bins[at * FINE + i] = (double)bins[i];
}

struct Chosen {
    uint64_t tokens[MOST];   // key, then the index's complement: falling, the lowest index first
    uint32_t counts[FINE], starts[FINE];
    uint64_t kept[MOST_PARTS];
    double factor[MOST_PARTS];  // of a part's weights in the row's unit
    int away[MOST_PARTS];       // bins between its largest logit and the row's
    uint64_t part[WAVES];
    uint32_t count, low, crowded;
    int found;
    uint64_t before;
};
union RowShared {
    WholeRow whole;
    Chosen chosen;
};

// sum of x over the threads before this one; `all`: over all threads
SAMPLE_DEV uint64_t sum_before(uint64_t x, uint64_t* part, uint64_t& all) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint64_t s = wave_upto(x);
    __syncthreads();
    if (lane == 63) part[wave] = s;
    __syncthreads();
    const uint64_t w = row_upto(part[lane % WAVES]);
    all = lane_of(w, WAVES - 1);
    return (wave ? lane_of(w, wave - 1) : 0) + s - x;
}
// Sorts n different tokens, falling: into 1024 bins of equal width by value(token), which orders them the same way and is below `range`, and within a bin
// by counting the larger ones.  EACH: tokens of a thread; false: too many in a bin.
template <int EACH, class V> SAMPLE_DEV bool sort_by_bins(Chosen& sh, int n, V value, uint64_t range) {
    uint64_t *const v = sh.tokens, own[EACH];
    uint32_t slot[EACH];
    int bin[EACH];
    sh.counts[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.crowded = 0;
    const float scale = 1023.0f / (float)range;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int i = threadIdx.x + e * THREADS;
        own[e] = i < n ? v[i] : 0;
        bin[e] = i < n ? min((int)((float)(range - 1 - value(own[e])) * scale), FINE - 1) : 0;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < EACH; ++e)
        if ((int)threadIdx.x + e * THREADS < n) {
            slot[e] = atomicAdd(&sh.counts[bin[e]], 1u);
            if (slot[e] >= 48) sh.crowded = 1;
        }
    __syncthreads();
    if (sh.crowded) return false;
    uint64_t all;
    sh.starts[threadIdx.x] = (uint32_t)sum_before(sh.counts[threadIdx.x], sh.part, all);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < EACH; ++e)
        if ((int)threadIdx.x + e * THREADS < n) v[sh.starts[bin[e]] + slot[e]] = own[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < EACH; ++e)
        if ((int)threadIdx.x + e * THREADS < n) {
            const uint32_t from = sh.starts[bin[e]], count = sh.counts[bin[e]];
            slot[e] = from;
            for (uint32_t j = 0; j < count; ++j) slot[e] += v[from + j] > own[e];
        }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < EACH; ++e)
        if ((int)threadIdx.x + e * THREADS < n) v[slot[e]] = own[e];
    __syncthreads();
    return true;
}
// The same whatever their bins: then by halves, where pairs up to 64 apart are one wavefront's.
template <class V> SAMPLE_DEV void sort(Chosen& sh, int n, V value, uint64_t range) {
    if (n <= THREADS ? sort_by_bins<1>(sh, n, value, range) : sort_by_bins<MOST / THREADS>(sh, n, value, range)) return;
    __syncthreads();
    uint64_t* const v = sh.tokens;
    int to = 64;
    while (to < n) to *= 2;
    for (int i = n + threadIdx.x; i < to; i += THREADS) v[i] = 0;  // zeros sort last
    __syncthreads();
    for (int k = 2; k <= to; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            if (j >= 64) __syncthreads();
            for (int t = threadIdx.x; t < to / 2; t += THREADS) {
                const int i = 2 * t - (t & (j - 1));
                const uint64_t x = v[i], y = v[i + j];
                if ((x < y) == ((i & k) == 0)) v[i] = y, v[i + j] = x;
            }
            if (j >= 64) __syncthreads();
            else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    __syncthreads();
}
SAMPLE_DEV uint32_t key_in(uint64_t token) { return (uint32_t)(token >> 32); }
SAMPLE_DEV int index_in(uint64_t token) { return (int)~(uint32_t)token; }

struct Result {  // of the thread that finds the token
    int token = -1;
    double log_weight = 0.0;
    uint64_t all = 1;
};

// The row as a whole, from its logits alone.
template <int DT> SAMPLE_DEV void whole_row(const SampleArgs& a, WholeRow& sh, const uint8_t* row, const Limits& l, const Weights& weights, Result& found) {
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
        const uint64_t upto = before + wave_upto(w);
        const uint64_t over = __ballot(upto > target);
        if (over) {
            if (lane == __ffsll((unsigned long long)over) - 1) found = {i, x, total};
            return;
        }
        before = shfl(upto, 63);
        ties_before += (uint32_t)__popcll(equals);
    }
}

// Collects the tokens whose logits are from `low` to `high`; there may be more than MOST.
template <int DT> SAMPLE_DEV void collect(const SampleArgs& a, Chosen& sh, const uint8_t* row, float low, float high) {
    constexpr int AHEAD = DT == OGC_F32 ? 4 : 8;  // chunks of a thread whose loads are on their way together
    const float* const tops = a.tops + (int64_t)blockIdx.x * a.chunks;
    const int off = off_of<DT>(row);
    low = fmaxf(low, -3.4028234663852886e38f);  // (minus infinity is no token)
    float after[AHEAD];
    const auto look = [&](int i0) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) after[u] = tops[min(i0 + u * THREADS, a.chunks - 1)];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) after[u] = i0 + u * THREADS < a.chunks ? after[u] : -INFINITY;
    };
    look(threadIdx.x);
#pragma unroll 1
    for (int i0 = threadIdx.x; i0 < a.chunks; i0 += AHEAD * THREADS) {
        float m[AHEAD];
        Eight<DT> x[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) m[u] = after[u];
        look(i0 + AHEAD * THREADS);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int i = (i0 + u * THREADS) * 8 - off;
            if (m[u] >= low && i >= 0 && i + 8 <= a.vocab) x[u].whole(row, i);
        }
#pragma unroll
        for (int g = 0; g < AHEAD; g += 4) {  // (four chunks, a bit a token: put away together, since a wavefront goes on until its last lane has done so)
            uint32_t pass = 0;
#pragma unroll
            for (int u = g + 3; u >= g; --u) {
                uint32_t of_chunk = 0;
                if (m[u] >= low) {
                    const int i = (i0 + u * THREADS) * 8 - off;
                    if (i < 0 || i + 8 > a.vocab) x[u].part(row, i, a.vocab);
#pragma unroll
                    for (int e = 0; e < 8; ++e) of_chunk |= x[u].get(e) >= low && x[u].get(e) <= high ? 1u << e : 0u;
                }
                pass = pass << 8 | of_chunk;
            }
            if (!pass) continue;
            uint32_t to = atomicAdd(&sh.count, (uint32_t)__popc(pass));
            for (; pass; pass &= pass - 1, ++to) {
                const int bit = __ffs(pass) - 1;
                if (to < MOST) sh.tokens[to] = (uint32_t)((i0 + (g + bit / 8) * THREADS) * 8 - off + bit % 8);
            }
        }
    }
    __syncthreads();
    const int n = min((int)sh.count, MOST);
    for (int j = threadIdx.x; j < n; j += THREADS) {  // (the logits once more: all at once, where picking them out above would be one after the other)
        const uint32_t i = (uint32_t)sh.tokens[j];
        sh.tokens[j] = (uint64_t)key_of(logit_at<DT>(row, (int)i)) << 32 | ~i;
    }
    __syncthreads();
}
// The key of the least logit whose place is `place` or more (a whole number, 2^23 at most from 0); -0 and 0 have keys of their own here.
SAMPLE_DEV uint32_t first_at(float place, float fine) {
    uint32_t low = 0x00800000u, high = 0xff7fffffu;  // keys: of the least fp32 number, of the largest
    const float x = place / fine;
    const uint32_t near = key_of(x);
    if (__builtin_fabsf(x) < 0x1p120f && near > low + 16 && near < high - 16) {  // (a quotient is hardly off: most of the way at once)
        if (place_of(logit_of(near + 8), fine) >= place) high = near + 8;
        if (!(place_of(logit_of(near - 8), fine) >= place)) low = near - 7;
    }
    while (low < high) {
        const uint32_t mid = low + (high - low) / 2;
        if (place_of(logit_of(mid), fine) >= place) high = mid;
        else low = mid + 1;
    }
    return low;
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

// Sorts tokens whose keys are from least to most by their logits, the lowest index first of equal ones: by logit and index together, counted in the steps that
// the type has, so that equal logits (in bf16 there are many) do not share a bin.
template <int DT> SAMPLE_DEV void sort_by_logit(Chosen& sh, int n, int vocab, uint32_t least, uint32_t most) {
    constexpr int STEP = DT == OGC_F32 ? 0 : 16;
    sort(sh, n, [&](uint64_t t) { return (uint64_t)((key_in(t) >> STEP) - (least >> STEP)) * vocab + (vocab - 1 - index_in(t)); },
         (uint64_t)((most >> STEP) - (least >> STEP) + 1) * vocab);
}

// The choice among the first n <= 1024 tokens, which become sorted by index.
SAMPLE_DEV Result choose(Chosen& sh, int n, int vocab, const Weights& weights, float u) {
    if ((int)threadIdx.x < n) sh.tokens[threadIdx.x] = sh.tokens[threadIdx.x] << 32 | sh.tokens[threadIdx.x] >> 32;  // the index's complement first: falling is the lowest index first
    __syncthreads();
    sort(sh, n, [&](uint64_t t) { return (uint64_t)((uint32_t)(t >> 32) + (uint32_t)vocab); }, (uint64_t)vocab);  // (~index + vocab)
    const uint64_t mine = (int)threadIdx.x < n ? sh.tokens[threadIdx.x] : 0;
    const double x = (int)threadIdx.x < n ? weights.log_of(logit_of((uint32_t)mine)) : -INFINITY;
    const uint64_t w = Weights::of_log(x);
    uint64_t all;
    const uint64_t run = sum_before(w, sh.part, all), target = target_of(u, all);
    Result found;
    if (run <= target && target < run + w) found = {(int)~(uint32_t)(mine >> 32), x, all};
    return found;
}

// How many of the first n sorted tokens are kept by top-p and min-p; `before`: the weight ahead of them; `goal`: top-p's, or 0: its share of these tokens' weight.
template <int EACH> SAMPLE_DEV int kept_of(Chosen& sh, int n, const Weights& weights, const Limits& l, uint64_t before, uint64_t goal) {  // EACH: tokens of a thread
    if (threadIdx.x == 0) sh.found = n;
    uint64_t w[EACH], own = 0;
    double x[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int i = threadIdx.x * EACH + e;
        x[e] = i < n ? weights.log_of(logit_of(key_in(sh.tokens[i]))) : -INFINITY;
        w[e] = Weights::of_log(x[e]);
        own += w[e];
    }
    uint64_t all, run = before + sum_before(own, sh.part, all);
    if (goal == 0) goal = goal_of(l.p, all);
    int mine = n;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int i = threadIdx.x * EACH + e;
        if (i < mine && (w[e] == 0 || (l.top_p && run >= goal) || !(x[e] >= l.least))) mine = i;
        run += w[e];
    }
    if (mine < n) atomicMin(&sh.found, mine);
    __syncthreads();
    return sh.found;
}

// A row's choice by top-k, and then the other limits; false: nothing was chosen.
template <int DT> SAMPLE_DEV bool by_top_k(const SampleArgs& a, Chosen& sh, const uint8_t* row, const Limits& l, const Weights& weights, float high, float u, int r, Result& found) {
    const float* const tops = a.tops + (int64_t)r * a.chunks;
    const auto away = [&](float x) { return high - place_of(x, l.fine); };
    // ---- the bin of the k-th of 2048 largest logits, two a thread (of 1024 the thousandth would have some four thousand tokens before it)
    sh.counts[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.count = 0, sh.low = 0xffffffffu, sh.found = FINE;
    float m[2] = {-INFINITY, -INFINITY}, d[2];
#pragma unroll 1
    for (int i = threadIdx.x; i < a.chunks; i += 8 * THREADS) {
        float t[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) t[u] = tops[min(i + u * THREADS, a.chunks - 1)];
#pragma unroll
        for (int u = 0; u < 8; ++u) m[u % 2] = i + u * THREADS < a.chunks ? fmaxf(m[u % 2], t[u]) : m[u % 2];
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        d[h] = m[h] == -INFINITY ? (float)FINE : away(m[h]);
        if (d[h] < (float)FINE) atomicAdd(&sh.counts[(int)d[h]], 1u);
    }
    __syncthreads();
    uint64_t all;
    const uint64_t c = sh.counts[threadIdx.x], s = sum_before(c, sh.part, all), k = (uint64_t)l.k;
    if (s < k && k <= s + c) sh.found = threadIdx.x;
    __syncthreads();
    // the smallest of those up to that bin: k tokens at least are as large.  (Fewer than k with a weight: all that have one.)
    const bool enough = sh.found < FINE;
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (enough && d[h] <= (float)sh.found) atomicMin(&sh.low, key_of(m[h]));
    __syncthreads();
    const uint32_t low = enough ? sh.low : first_at(high - (float)(FINE - 1), l.fine);
    collect<DT>(a, sh, row, logit_of(low), INFINITY);
    int n = (int)sh.count;
    __syncthreads();
    if (n > MOST) return false;
    sort_by_logit<DT>(sh, n, a.vocab, min(low, key_of(logit_of(low))), key_of((float)weights.largest));
    n = min(n, l.k);
    if (l.top_p || l.min_p) n = kept_of<1>(sh, n, weights, l, 0, 0);
    found = choose(sh, n, a.vocab, weights, u);
    return true;
}

// A row's choice by top-p and min-p, or without limits; false: nothing was chosen.
template <int DT> SAMPLE_DEV bool by_parts(const SampleArgs& a, Chosen& sh, const uint8_t* row, const Limits& l, const Weights& weights, float high, float u, int r, Result& found) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool limited = l.top_p || l.min_p;
    const float* const largest = a.largest + (int64_t)r * a.parts;
    const uint64_t* const mass = a.mass + (int64_t)r * a.parts;
    const double* const bins = a.bins + (int64_t)r * a.parts * FINE;
    const auto away = [&](float x) { return high - place_of(x, l.fine); };
    if ((int)threadIdx.x < a.parts) {
        const float m = largest[threadIdx.x];
        const double f = m == (float)weights.largest ? 1.0 : exp(((double)m - weights.largest) * l.per);
        const float d = away(m);
        sh.factor[threadIdx.x] = f > 0.0 ? f : 0.0;
        sh.away[threadIdx.x] = m > -INFINITY && d < (float)FINE ? (int)d : FINE;
    }
    if (threadIdx.x == 0) sh.count = 0, sh.found = FINE - 1;
    __syncthreads();
    const auto in_row = [&](uint64_t mass, int p) { return (uint64_t)((double)mass * sh.factor[p]); };
    int from = FINE, kept = 0;  // kept: all of the bins before `from`, and the first `kept` sorted tokens
    if (limited) {
        // ---- bins of the row, a thread each
        double of_bin = 0.0;  // (the parts always one after the other)
#pragma unroll 1
        for (int p0 = 0; p0 < a.parts; p0 += 8) {
            double b[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {  // (a part of no use is a whole row of bins away)
                const int p = min(p0 + u, a.parts - 1);
                b[u] = bins[(int64_t)p * FINE + max((int)threadIdx.x - sh.away[p], 0)];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (p0 + u < a.parts && (int)threadIdx.x >= sh.away[p0 + u]) of_bin += b[u] * sh.factor[p0 + u];
        }
        const uint64_t b = (uint64_t)of_bin;
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
        // (up to the last logit that is not in the bins before)
        const uint32_t low = first_at(high - (float)to, l.fine), behind = from ? first_at(high - (float)(from - 1), l.fine) - 1 : key_of((float)weights.largest);
        collect<DT>(a, sh, row, logit_of(low), from ? logit_of(behind) : INFINITY);
        const int n = (int)sh.count;
        __syncthreads();
        if (n > MOST) return false;
        sort_by_logit<DT>(sh, n, a.vocab, min(low, key_of(logit_of(low))), max(behind, key_of(logit_of(behind))));
        kept = n <= THREADS ? kept_of<1>(sh, n, weights, l, before, goal) : kept_of<MOST / THREADS>(sh, n, weights, l, before, goal);
    }
    // ---- the part that has the token: what is kept of each
    const int off = off_of<DT>(row);
    const uint64_t end = kept ? sh.tokens[kept - 1] : ~0ull;  // the last of the sorted tokens that are kept
    if ((int)threadIdx.x < a.parts) sh.kept[threadIdx.x] = limited ? 0 : in_row(mass[threadIdx.x], threadIdx.x);
    __syncthreads();
    for (int i = threadIdx.x; i < kept; i += THREADS)
        atomicAdd((unsigned long long*)&sh.kept[(index_in(sh.tokens[i]) + off) / a.part], (unsigned long long)weights.of(key_in(sh.tokens[i])));
    if (limited)
        for (int p = wave; p < a.parts; p += WAVES) {
            const int count = from - sh.away[p];
            if (count <= 0) continue;
            double m = 0.0;
#pragma unroll 8
            for (int i = lane; i < count; i += 64) m += bins[(int64_t)p * FINE + i];
            const uint64_t here = wave_sum((uint64_t)m);
            if (lane == 0) atomicAdd((unsigned long long*)&sh.kept[p], (unsigned long long)in_row(here, p));
        }
    __syncthreads();
    const uint64_t own = (int)threadIdx.x < a.parts ? sh.kept[threadIdx.x] : 0;
    uint64_t total, run = sum_before(own, sh.part, total);
    const uint64_t target = target_of(u, total);
    if (run <= target && target < run + own) sh.found = threadIdx.x, sh.before = run;
    __syncthreads();
    // ---- its tokens, in the part's own unit
    const int p = sh.found;
    const double rest = (double)(target - sh.before) / sh.factor[p];
    Weights near = weights;
    near.largest = largest[p];
    const int at = p * a.part + (int)threadIdx.x * 8 - off;
    Eight<DT> x;
    if ((int)threadIdx.x * 8 < a.part) x.load(row, at, a.vocab);
    else x.clear();
    const auto weight = [&](float v, int e) -> uint64_t {
        const uint64_t token = (uint64_t)key_of(v) << 32 | (uint32_t)~(uint32_t)(at + e);
        if (!(v > -INFINITY) || (limited && !(away(v) < (float)from) && token < end)) return 0;
        return near.largest == INFINITY ? Weights::of_infinite(v) : near.of_part(v);
    };
    uint64_t mine = 0, all;
#pragma unroll 4
    for (int e = 0; e < 8; ++e) {
        mine += weight(x.get(0), e);
        x.next();
    }
    run = sum_before(mine, sh.part, all);
    const uint64_t goal = rest < (double)all && (uint64_t)rest < all ? (uint64_t)rest : all - 1;
    if (run <= goal && goal < run + mine) {
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
            const uint64_t w = weight(x.get(0), e);
            if (goal < run + w) {
                found = {at + e, weights.log_of(x.get(0)), total};
                break;
            }
            run += w;
            x.next();
        }
    }
    return true;
}

// ---- the choice, a workgroup for each row.  Bound by the latency of its steps (32000 bf16 logits with all limits 12.5 us: the limit of top-k 2, collecting 4, sorting 2,
// what top-p and min-p keep 2, the choice 2), for long flat rows by a compute unit's way through their chunks (64 x 128000, top-p 30.8 us, 11 of them collecting).
template <int DT> __global__ __launch_bounds__(THREADS) void ogc_sample_kernel(SampleArgs a) {
    __shared__ RowShared shared;
    Chosen& sh = shared.chosen;
    const int lane = threadIdx.x & 63, r = blockIdx.x;
    const uint8_t* const row = a.logits + r * a.stride;
    const Limits l = limits_of(a, r);
    const float u = a.uniform[r];
    float top = -INFINITY;
    for (int i = lane; i < a.parts; i += 64) top = fmaxf(top, a.largest[(int64_t)r * a.parts + i]);
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
        const float* const tops = a.tops + (int64_t)r * a.chunks;
        if (threadIdx.x == 0) sh.found = 0x7fffffff;
        __syncthreads();
        for (int i = threadIdx.x; i < a.chunks; i += THREADS)
            if (tops[i] == top) {
                atomicMin(&sh.found, i);
                break;
            }
        __syncthreads();
        if (threadIdx.x == 0) {
            const int at = sh.found * 8 - off_of<DT>(row);
            Eight<DT> x;
            x.load(row, at, a.vocab);
            int first = 7;
#pragma unroll
            for (int e = 6; e >= 0; --e)
                if (x.get(e) == top) first = e;
            a.tokens[r] = at + first;
            if (a.logs) a.logs[r] = 0.0f;
        }
        return;
    }
    Weights weights;
    weights.largest = top;
    weights.per = l.per;
    const float high = place_of(top, l.fine);
    // places are whole numbers, and near enough to where the logits are, up to 2^22
    bool done = !(l.top_k || l.top_p || l.min_p) || (__builtin_fabsf(high) < 0x1p22f && (!l.top_k || l.k <= MOST_K));
    Result found;
    if (done) done = l.top_k ? by_top_k<DT>(a, sh, row, l, weights, high, u, r, found) : by_parts<DT>(a, sh, row, l, weights, high, u, r, found);
    if (!done) whole_row<DT>(a, shared.whole, row, l, weights, found);
    if (found.token >= 0) {
        a.tokens[r] = found.token;
        if (a.logs) a.logs[r] = (float)(found.log_weight - log((double)found.all * 0x1p-42));
    }
}

// Chunks and parts of a row that begins up to seven tokens behind a multiple of 16 bytes.
int chunks_of(const ogc_sample_desc* d) { return (d->vocab + 7 + 7) / 8; }
int parts_of(const ogc_sample_desc* d, int part) { return (d->vocab + 7 + part - 1) / part; }
// Tokens of a part: as many as leave the chip enough workgroups, 8192 at most; 256 parts of a row at most.
int part_of(const ogc_sample_desc* d) {
    int part = 8192;
    while (part > 2048 && (int64_t)d->rows * parts_of(d, part) < 512 && parts_of(d, part / 2) <= MOST_PARTS) part /= 2;
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
    const size_t part = (size_t)part_of(d), parts = parts_of(d, (int)part), chunks = chunks_of(d);
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
    a.parts = parts_of(d, a.part);
    a.chunks = chunks_of(d);
    a.bins = (double*)workspace;
    a.mass = (uint64_t*)a.bins + (size_t)d->rows * a.parts * FINE;
    a.largest = (float*)(a.mass + (size_t)d->rows * a.parts);
    a.tops = a.largest + (size_t)d->rows * a.parts;
    const hipStream_t s = (hipStream_t)stream;
    if (d->dtype == OGC_F32) launch<OGC_F32>(a, s);
    else launch<OGC_BF16>(a, s);
    return hipGetLastError() == hipSuccess ? OGC_OK : OGC_ERR_DEVICE;
}

}  // extern "C"
