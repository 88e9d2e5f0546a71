// Attention of a few queries of each sequence over the 4-bit cache (include/ogc_decoder.h).
//
// A sequence's queries times the query heads of a key head are the columns of a tile of 16; a wavefront takes 32 tokens of the cache
// (a record) at a time and keeps its columns' running maxima, sums and outputs in registers.  Both products are
// transposed (16x16x32 matrix instruction, operands: row or column = lane % 16, k = 8 * (lane / 16) ..; results: column = lane % 16,
// rows 4 * (lane / 16) ..), and the record's layout hands every lane its operand in whole dwords:
//
//   S^T[token][column] = K Q^T    a lane has the channels d/4 * (lane / 16) .. of one token (the queries' channels in the same order);
//                                 codes become bf16 values with their scale in one conversion.  Row m of tile b is token
//                                 8 (m / 4) + 4 b + m % 4, which leaves a lane with the tokens 8 * (lane / 16) ..: just
//                                 those whose weights the second product wants from it.
//   O^T[channel][column] += V^T P^T   a dword is one channel's values of eight tokens.  Their scales differ by token, so they
//                                 go into the weights, for each 32 channels (a power of two: nothing is rounded by it).
//
// The weights carry a factor 2^30, which the division takes out again: with the smallest scales they keep all their digits.  With
// scales from some 2^80 on their sums may overflow: a workgroup that finds one that is not finite computes its share once more with a factor
// that all its tokens cannot overflow, and takes from that what was not finite (the other channels may hold the smallest values).
// A scale of no number (byte 255) becomes an infinity here, and what is not finite even then becomes NaN: values of the cache are finite
// otherwise, and so are their weighted means.  Splits are joined as means, too: their sums might overflow once more.
#include "ogc_attention.h"
#include "ogc_decoder.h"
#include "ogc_kv4_host.h"
#include "ogc_kv4_layout.h"

namespace {

typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v3u __attribute__((ext_vector_type(3)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

struct StepArgs {
    const uint8_t* q;
    const uint8_t* cache;
    uint8_t* o;
    const int32_t* cu;
    const int32_t* lens;
    const int32_t* table;
    float* partial;  // [split][row][head][d], then the maxima and sums [split][row][head][2]
    float* stats;
    long long sq[2], so[2];  // bytes: row, head
    int rows, max_rows, max_keys;
    int heads, group;  // key heads, query heads of each
    int page_size, pages, width;
    int chunk, splits, columns;  // tokens of a split (a multiple of 32 times the wavefronts), splits of the longest, workgroups along the columns
    float scale_log2;
};

// one sequence's share of a launch, the same in both kernels
struct StepSequence {
    int row0, n, len, off;  // query i sees the tokens up to i + off
};
__device__ __forceinline__ StepSequence sequence_of(const StepArgs& a, int b) {
    StepSequence s;
    s.row0 = min(max(a.cu[b], 0), a.rows);
    const int n = min(max(a.cu[b + 1], s.row0), a.rows) - s.row0;
    s.n = min(n, a.max_rows);
    s.len = min(max(a.lens[b], 0), a.max_keys);  // (the host holds max_keys to the table's tokens)
    s.off = s.len - n;
    return s;
}

// N dwords of LDS, aligned to what is a power of two of them
template <int N> struct Dwords {
    typedef uint32_t type __attribute__((ext_vector_type(N)));
    static __device__ __forceinline__ uint32_t at(const type& x, int i) { return x[i]; }
    static __device__ __forceinline__ type load(const uint8_t* p) { return *(const type*)p; }
};
template <> struct Dwords<1> {
    typedef uint32_t type;
    static __device__ __forceinline__ uint32_t at(type x, int) { return x; }
    static __device__ __forceinline__ type load(const uint8_t* p) { return *(const uint32_t*)p; }
};
template <> struct Dwords<3> {
    typedef v3u type;
    static __device__ __forceinline__ uint32_t at(const type& x, int i) { return x[i]; }
    static __device__ __forceinline__ type load(const uint8_t* p) { return (v3u){((const uint32_t*)p)[0], ((const uint32_t*)p)[1], ((const uint32_t*)p)[2]}; }
};

// eight codes as an operand, times a power of two (the exponent's bits of `scale`)
__device__ __forceinline__ v8bf operand(uint32_t codes, float scale) {
    const v2bf x0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    const v2bf x2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), x3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return (v8bf){x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
}
// the value of byte i of a pair of dwords as an fp32 exponent
__device__ __forceinline__ float exponent(const v2u& x, int i) {
    return __builtin_bit_cast(float, (x[i / 4] >> (8 * (i % 4)) & 255u) << 23);
}
// the square root of 2^x, to be multiplied by twice: the power itself ends at 2^-126, although what it is multiplied by carries 2^30, and a
// channel may have nothing but a value that small
__device__ __forceinline__ float half_power(float x) { return __builtin_amdgcn_exp2f(0.5f * x); }
__device__ __forceinline__ v4f mma(const v8bf& x, const v8bf& y, const v4f& z) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, z, 0, 0, 0); }

// The records of a run of tokens, one after the other, all arithmetic the same for a whole wavefront.
struct RecordWalk {
    typedef const __attribute__((address_space(4))) int32_t* Entries;  // (constant memory: a scalar load, which the counted ones do not wait for)
    Entries entries;
    const uint8_t* heads;  // the cache's first record of this head
    int64_t page_bytes;
    int page_records, pages, entry, at;  // at: record inside the page
    __device__ __forceinline__ void start(const StepArgs& a, int b, int head, int d, int token) {
        page_records = a.page_size / KV4_TOKENS;
        page_bytes = (int64_t)a.heads * page_records * kv4_record_bytes(d);
        heads = a.cache + (int64_t)head * page_records * kv4_record_bytes(d);
        entries = (Entries)(uintptr_t)(a.table + (int64_t)b * a.width);
        pages = a.pages;
        entry = token / a.page_size;
        at = token % a.page_size / KV4_TOKENS;
    }
    // the record that the walk is at (the caller has seen to it that it is one of the table's), or nullptr where there is no page; then one further
    __device__ __forceinline__ const uint8_t* next(int d) {
        const int page = entries[entry];
        const uint8_t* r = page < 0 || page >= pages ? nullptr : heads + page * page_bytes + (int64_t)at * kv4_record_bytes(d);
        if (++at == page_records) {
            at = 0;
            ++entry;
        }
        return r;
    }
};

// Wavefronts on a SIMD that the registers are held to.
constexpr int step_waves(int dt, int t, int w) { return w == 8 || dt == OGC_F32 || t == 2 ? 2 : 3; }
constexpr int STEP_SLOTS = 3;  // records of a wavefront in LDS: the one in use and two on their way

// DT: of the queries.  T: column tiles of a wavefront.  W: wavefronts, which take the records of the split in turn.
template <int DT, int D32, int T, int W> __global__ __launch_bounds__(64 * W, step_waves(DT, T, W)) void ogc_kv4_attention_kernel(StepArgs a) {
    constexpr int D = D32 * 32, E = DT == OGC_F32 ? 4 : 2, P = DT == OGC_F32 ? 3 : 1, ROW = D + 4;
    constexpr int BYTES = 34 * D, RING = W * STEP_SLOTS * BYTES, JOIN = W * 16 * ROW * 4;
    __shared__ float stat_lds[2][W][16 * T];
    __shared__ __attribute__((aligned(16))) uint8_t lds[RING > JOIN ? RING : JOIN];
    float(*const o_lds)[16][ROW] = (float(*)[16][ROW])lds;
    const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.y;
    const uint32_t x = blockIdx.x;
    const int head = x % (uint32_t)a.heads, y = x / (uint32_t)a.heads, split = y / (uint32_t)a.columns, c0 = y % (uint32_t)a.columns * 16 * T;
    const StepSequence s = sequence_of(a, b);
    const int k0 = split * a.chunk;  // (below max_keys)
    if (c0 >= s.n * a.group || (split > 0 && k0 >= s.len)) return;
    const int k1 = kv4_split_end(s.len, a.chunk, k0);

    // ---- queries: the second operand of the first product, in one or three bf16 pieces.  Three pieces hold an fp32 value from 2^-110 on, and below
    // bf16's largest: a query whose largest channel is below 2^-46 or from 2^64 on is multiplied by a power of two, which its scores' scale takes out
    // again, so that only channels 2^-64 times that large can lose digits.
    v8bf q[T][P][D32];
    float by[T];  // the scores' scale, base-2 logarithms
    int limit[T];  // the last token that this lane's column sees
    float ref[T], sum[T];
    v4f out[T][D32][2];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int c = c0 + 16 * t + col, i = c / (uint32_t)a.group;
        const bool on = i < s.n;
        limit[t] = on ? s.off + i : -1;
        const uint8_t* p = a.q + (long long)(s.row0 + (on ? i : 0)) * a.sq[0] + (long long)(head * a.group + c - i * a.group) * a.sq[1] + g * D32 * 8 * E;
        by[t] = a.scale_log2;
        if constexpr (P == 1) {
            const v4i z = {0, 0, 0, 0};
#pragma unroll
            for (int d = 0; d < D32; ++d) q[t][0][d] = __builtin_bit_cast(v8bf, on ? *(const v4i*)(p + d * 16) : z);
        } else {
            const v4f z = {0.0f, 0.0f, 0.0f, 0.0f};
            v4f x[2 * D32];
            float most = 0.0f;
#pragma unroll
            for (int d = 0; d < 2 * D32; ++d) {
                x[d] = on ? *(const v4f*)(p + d * 16) : z;
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, fabsf(x[d][e]));
            }
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            const float up = most < 0x1p-46f ? 0x1p64f : most >= 0x1p64f ? 0x1p-64f : 1.0f;
            by[t] *= most < 0x1p-46f ? 0x1p-64f : most >= 0x1p64f ? 0x1p64f : 1.0f;
#pragma unroll
            for (int d = 0; d < D32; ++d) {
                const Pieces8 r = split8(x[2 * d] * up, x[2 * d + 1] * up);
#pragma unroll
                for (int i = 0; i < 3; ++i) q[t][i][d] = __builtin_bit_cast(v8bf, r.p[i]);
            }
        }
    }
    const int first_limit = s.off + c0 / (uint32_t)a.group;  // of the first column: the least

    // ---- the records of this wavefront: neighbours.  They go straight into LDS, two ahead of their use, by loads that hold no registers: a
    // record is 17 lines of 256 bytes for 128 channels, and the chip needs some 50 KiB of them on their way to every compute unit.
    const int records = (k1 - k0 + KV4_TOKENS - 1) / KV4_TOKENS, each = (records + W - 1) / W;
    const int first = k0 + wave * each * KV4_TOKENS, end = min(k1, first + each * KV4_TOKENS);
    const int count = max((end - first + KV4_TOKENS - 1) / KV4_TOKENS, 0);
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds + wave * (STEP_SLOTS * BYTES);
    constexpr int LOADS = D32 + 1;  // of a record: 1 KiB each, and the exponents
    const uint32_t piece = lane * 16;
    auto issue = [&](const uint8_t* r, int slot) {
        const uint32_t to = __builtin_amdgcn_readfirstlane(ring + slot * BYTES);
#pragma unroll
        for (int i = 0; i < D32; ++i)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to + i * 1024), "v"(piece), "s"(r + i * 1024) : "memory", "m0");
        if (lane < D / 8)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to + D32 * 1024), "v"(piece), "s"(r + D32 * 1024) : "memory", "m0");
    };
    float factor = 30.0f;  // of the weights, base-2 logarithm
    uint32_t bad = 0;      // of this thread's outputs (see below), those that were not finite with it
again:
#pragma unroll
    for (int t = 0; t < T; ++t) {
        ref[t] = -INFINITY;
        sum[t] = 0.0f;
#pragma unroll
        for (int d = 0; d < D32; ++d) out[t][d][0] = out[t][d][1] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
    }
    RecordWalk walk;
    walk.start(a, b, head, D, first);
    uint32_t there = 0;  // bit i: there is a page for the record i ahead.  (Where there is none, the cache's first record is loaded: loads are counted.)
    auto fetch = [&](int i) {
        const uint8_t* r = walk.next(D);
        there |= (r ? 1u : 0u) << (STEP_SLOTS - 1);
        issue(r ? r : a.cache, i % STEP_SLOTS);
    };
    for (int i = 0; i < STEP_SLOTS - 1; ++i) {
        if (i < count) fetch(i);
        there >>= 1;
    }
    for (int i = 0; i < count; ++i) {
        const int token = first + i * KV4_TOKENS;
        // what was read of the slot that is loaded now has been read; then all but the newest loads have landed
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (i + STEP_SLOTS - 1 < count) {
            fetch(i + STEP_SLOTS - 1);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STEP_SLOTS - 1) * LOADS) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        const bool here = there & 1;
        there >>= 1;
        if (!here) continue;
        const uint8_t* const r = lds + wave * (STEP_SLOTS * BYTES) + i % STEP_SLOTS * BYTES;
        const bool whole = token + KV4_TOKENS - 1 <= first_limit;

        v4f sc[T][2];
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) {
            v8bf k[D32];
            const int key = 8 * (col / 4) + 4 * tile + col % 4;
            const typename Dwords<D32>::type codes = Dwords<D32>::load(r + kv4_key_at(D, key, 8 * D32 * g));
#pragma unroll
            for (int d = 0; d < D32; ++d)  // (a lane's channels have one scale, for 96 of them up to three)
                k[d] = operand(Dwords<D32>::at(codes, d), __builtin_bit_cast(float, (uint32_t)r[kv4_key_scale_at(D, (D32 * g + d) / 4, key)] << 23));
#pragma unroll
            for (int t = 0; t < T; ++t) {
                v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
                // (the instruction truncates what it adds to a larger sum: small products first)
#pragma unroll
                for (int d = 0; d < D32; ++d)
#pragma unroll
                    for (int p = P - 1; p > 0; --p) acc = mma(k[d], q[t][p][d], acc);
#pragma unroll
                for (int d = 0; d < D32; ++d) acc = mma(k[d], q[t][0][d], acc);
                sc[t][tile] = acc;
            }
        }
        float e[T][8];  // scores, then weights, of this lane's eight tokens
        v2u see[T];     // ones in the bytes of those that the column sees
#pragma unroll
        for (int t = 0; t < T; ++t) {
            // ---- tokens 8 g + j
            float cand = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                e[t][j] = sc[t][j >> 2][j & 3];
                cand = fmaxf(cand, e[t][j]);
            }
            see[t] = (v2u){~0u, ~0u};
            if (!whole) {  // tokens that the column does not see: their scores, and the exponents of their values, whatever stands there
                asm volatile("");  // (a branch, not forty selections in every record)
                cand = -INFINITY;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool hidden = token + 8 * g + j > limit[t];
                    e[t][j] = hidden ? -INFINITY : e[t][j];
                    see[t][j / 4] &= hidden ? ~(255u << (8 * (j % 4))) : ~0u;
                    cand = fmaxf(cand, e[t][j]);
                }
            }
            cand *= by[t];  // (positive)
            // The reference of the exponentials only has to be near the maximum: it moves where a block exceeds it by 2^8.
            if (__builtin_amdgcn_ballot_w64(cand > ref[t] + 8.0f) != 0) {
                cand = fmaxf(cand, __shfl_xor(cand, 16));
                cand = fmaxf(cand, __shfl_xor(cand, 32));
                const float to = fmaxf(ref[t], cand), half = to == -INFINITY ? 1.0f : half_power(ref[t] - to);
                ref[t] = to;
                sum[t] = sum[t] * half * half;
#pragma unroll
                for (int d = 0; d < D32; ++d)
#pragma unroll
                    for (int h = 0; h < 2; ++h) out[t][d][h] = out[t][d][h] * half * half;
            }
            const float off = ref[t] == -INFINITY ? 0.0f : factor - ref[t];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[t][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(e[t][j], by[t], off));
            if constexpr (P == 1) {  // rounded once; the sum takes what the second product multiplies
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const uint32_t pr = pack_bf16(e[t][j], e[t][j + 1]);
                    sum[t] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, pr), (v2bf){(__bf16)1.0f, (__bf16)1.0f}, sum[t], false);
                    e[t][j] = __builtin_bit_cast(float, pr << 16);
                    e[t][j + 1] = __builtin_bit_cast(float, pr & 0xffff0000u);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[t] += e[t][j];
            }
        }
        // ---- O^T += V^T P^T, 32 channels at a time: the weights times the scales of their values, then two instructions
#pragma unroll
        for (int d = 0; d < D32; ++d) {
            v8bf w[T][P];
            const v2u scales = *(const v2u*)(r + kv4_value_scale_at(D, d, 8 * g)), codes = *(const v2u*)(r + kv4_value_at(D, g, 32 * d + col));
#pragma unroll
            for (int t = 0; t < T; ++t) {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = e[t][j] * exponent(scales & see[t], j);
                if constexpr (P == 1) {
                    const v4i r = {(int)upper_halves(f[0], f[1]), (int)upper_halves(f[2], f[3]), (int)upper_halves(f[4], f[5]), (int)upper_halves(f[6], f[7])};
                    w[t][0] = __builtin_bit_cast(v8bf, r);
                } else {
                    const Pieces8 r = split8((v4f){f[0], f[1], f[2], f[3]}, (v4f){f[4], f[5], f[6], f[7]});
#pragma unroll
                    for (int p = 0; p < 3; ++p) w[t][p] = __builtin_bit_cast(v8bf, r.p[p]);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const v8bf v = operand(codes[h], 1.0f);
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    if constexpr (P == 1) {
                        out[t][d][h] = mma(v, w[t][0], out[t][d][h]);
                    } else {  // a record's sum by itself, small products first
                        v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int p = 2; p >= 0; --p) acc = mma(v, w[t][p], acc);
                        out[t][d][h] += acc;
                    }
                }
            }
        }
    }

    // ---- the wavefronts' shares together
    constexpr int ROUNDS = (16 * D / 4 + 64 * W - 1) / (64 * W);  // a thread has four outputs of a column tile in each
    static_assert(4 * T * ROUNDS <= 32, "a bit of `bad` for each of them");
    __syncthreads();  // (every wavefront is done with its records)
#pragma unroll
    for (int t = 0; t < T; ++t) {
        sum[t] += __shfl_xor(sum[t], 16);
        sum[t] += __shfl_xor(sum[t], 32);
        if (g == 0) {
            stat_lds[0][wave][16 * t + col] = ref[t];
            stat_lds[1][wave][16 * t + col] = sum[t];
        }
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
#pragma unroll
        for (int d = 0; d < D32; ++d)
#pragma unroll
            for (int h = 0; h < 2; ++h) *(v4f*)&o_lds[wave][col][32 * d + 16 * h + 4 * g] = out[t][d][h];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < ROUNDS; ++n) {
            const int u = threadIdx.x + 64 * W * n, bit = 4 * (ROUNDS * t + n);
            if (u >= 16 * D / 4) continue;
            const int cc = u / (D / 4), ch = u % (D / 4) * 4, c = c0 + 16 * t + cc, i = c / (uint32_t)a.group;
            if (i >= s.n) continue;
            float top = -INFINITY, total = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) top = fmaxf(top, stat_lds[0][w][16 * t + cc]);
            v4f r = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float m = stat_lds[0][w][16 * t + cc], h = m == -INFINITY ? 0.0f : half_power(m - top);
                // (a wavefront whose scores are all no numbers has a sum that is none, and no maximum)
                const float l = stat_lds[1][w][16 * t + cc];
                total += m == -INFINITY ? l : l * h * h;
                r += *(const v4f*)&o_lds[w][cc][ch] * h * h;
            }
            const int row = s.row0 + i, hd = head * a.group + c - i * a.group;
            const float inv = 1.0f / total;
            uint32_t write = 15;
            if (factor > 0.0f) {
#pragma unroll
                for (int e = 0; e < 4; ++e) bad |= (total == 0.0f || fabsf(r[e]) < INFINITY ? 0u : 1u) << (bit + e);
            } else {
                write = bad >> bit & 15u;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = total == 0.0f ? 0.0f : fabsf(r[e]) < INFINITY ? r[e] * inv : NAN;
            if (a.splits > 1) {  // the mean of the split, its reference and its sum without the factor
                const long long at = ((long long)split * a.rows + row) * (a.heads * a.group) + hd;
                float* p = a.partial + at * D + ch;
                if (write == 15u) *(v4f*)p = r;
                else
                    for (int e = 0; e < 4; ++e)
                        if (write >> e & 1u) p[e] = r[e];
                if (ch == 0 && factor > 0.0f) {
                    a.stats[2 * at] = top;
                    a.stats[2 * at + 1] = total * 0x1p-30f;
                }
            } else {
                uint8_t* p = a.o + (long long)row * a.so[0] + (long long)hd * a.so[1] + ch * E;
                const v2u two = {pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
                if (write == 15u) {
                    if constexpr (DT == OGC_F32) *(v4f*)p = r;
                    else *(v2u*)p = two;
                } else {
                    for (int e = 0; e < 4; ++e) {
                        if (!(write >> e & 1u)) continue;
                        if constexpr (DT == OGC_F32) ((float*)p)[e] = r[e];
                        else ((uint16_t*)p)[e] = (uint16_t)(two[e / 2] >> (16 * (e % 2)));
                    }
                }
            }
        }
        if (t + 1 < T) __syncthreads();
    }
    if (factor > 0.0f && __syncthreads_or(bad != 0)) {
        // weights up to 2^8 (the reference follows at that distance), values below 1.5 * 2^127, and all the share's tokens
        factor = -(8.0f + (float)(32 - __builtin_clz(max(k1 - k0, 1))));
        goto again;
    }
}

// The splits of a query and head together: a workgroup each, four channels a thread, LANES threads for them, which take the splits in turn.
template <int DT, int D> __global__ __launch_bounds__(256) void ogc_kv4_attention_join_kernel(StepArgs a) {
    constexpr int CH = D / 4, LANES = D == 96 ? 8 : 256 / CH;
    __shared__ float stat_lds[2][LANES];
    __shared__ __attribute__((aligned(16))) float o_lds[LANES][D];
    const StepSequence s = sequence_of(a, blockIdx.y);
    const uint32_t heads = a.heads * a.group;
    const int ch = threadIdx.x % CH * 4, lane = threadIdx.x / CH, hd = blockIdx.x % heads, i = blockIdx.x / heads;
    if (i >= s.n) return;
    const int n = kv4_splits_of(s.len, a.chunk);
    const long long at = (long long)(s.row0 + i) * heads + hd, step = (long long)a.rows * heads;
    float top = -INFINITY, total = 0.0f;
    v4f r = {0.0f, 0.0f, 0.0f, 0.0f};  // the mean so far
    constexpr int AHEAD = 4;  // splits on their way at a time
    for (int k0 = lane; k0 < n && lane < LANES; k0 += AHEAD * LANES) {
        float m[AHEAD], l[AHEAD];
        v4f x[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const long long p = at + min(k0 + k * LANES, n - 1) * step;
            m[k] = a.stats[2 * p];
            l[k] = a.stats[2 * p + 1];
            x[k] = *(const v4f*)(a.partial + p * D + ch);
        }
        // (sums of zero - no page, or nothing seen - have no maximum; neither have those that are no numbers)
        float to = top;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (k0 + k * LANES >= n) m[k] = -INFINITY, l[k] = 0.0f, x[k] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
            to = fmaxf(to, m[k]);
        }
        const float back = top == -INFINITY ? 1.0f : half_power(top - to), before = total * back * back;
        total = before;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const float h = m[k] == -INFINITY ? 1.0f : half_power(m[k] - to);
            l[k] = l[k] * h * h;
            total += l[k];
        }
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        r *= before * inv;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) r += x[k] * (l[k] * inv);
        top = to;
    }
    if (lane < LANES) {
        if (ch == 0) stat_lds[0][lane] = top, stat_lds[1][lane] = total;
        *(v4f*)&o_lds[lane][ch] = r;
    }
    __syncthreads();
    if (lane > 0) return;
    float w[LANES];
    for (int k = 0; k < LANES; ++k) top = fmaxf(top, stat_lds[0][k]);
    total = 0.0f;
#pragma unroll
    for (int k = 0; k < LANES; ++k) {
        const float m = stat_lds[0][k], h = m == -INFINITY ? 1.0f : half_power(m - top);
        w[k] = stat_lds[1][k] * h * h;
        total += w[k];
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    r = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < LANES; ++k) r += *(const v4f*)&o_lds[k][ch] * (w[k] * inv);
    uint8_t* p = a.o + (s.row0 + i) * a.so[0] + hd * a.so[1] + ch * (DT == OGC_F32 ? 4 : 2);
    if constexpr (DT == OGC_F32) *(v4f*)p = r;
    else *(v2u*)p = (v2u){pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
}

bool strides_ok(const int64_t s[2], int elt) { return s[0] >= 0 && s[1] >= 0 && s[0] * elt % 16 == 0 && s[1] * elt % 16 == 0; }

constexpr int STEP_GROUPS = 768, STEP_ALONE = 1024;

struct StepShape {
    int waves, tiles, columns, chunk, splits;
    size_t bytes;
};
// How a call is cut.  Columns: 16 or (bf16) 32 a workgroup.  Tokens: into as many splits as give the chip 768 workgroups, the three a compute unit
// that it holds at a time for 128 channels, of a record for each of four wavefronts at least.  (With 768 / 2048, us, batch x tokens, 32 heads over 8 of
// 128 channels: 64 x 8192 118 / 120, 32 x up to 4001 29.9 / 28.6, 1 x 4000 13.8 / 13.2; one of 30000 with 8 x 96 17.3 / 22.9.)  Up to 1024 tokens one
// workgroup of eight wavefronts has them all: no second launch (alone / shared, us, the same heads: 1 x 500 10.1 / 14.2, 1 x 1000 10.5 / 12.7,
// 1 x 1500 13.3 / 13.3, 1 x 2000 15.3 / 13.4, 4 x up to 2000 15.8 / 13.0; 4 heads of 32: 1 x 1000 9.4 / 12.6, 1 x 2000 10.5 / 12.7; fp32, 8
// heads of 96: 1 x 500 10.3 / 12.9, 1 x 1000 13.2 / 13.4, 1 x 1500 16.6 / 13.0).
StepShape shape_of(const ogc_kv4_desc* c, const ogc_kv4_attention_desc* d) {
    StepShape s;
    const int group = d->q_heads / c->kv_heads;
    const int max_rows = d->max_rows < d->rows ? d->max_rows : d->rows;
    const int64_t columns = (int64_t)max_rows * group;
    s.tiles = d->dtype == OGC_BF16 && columns > 16 ? 2 : 1;
    s.columns = (int)((columns + 16 * s.tiles - 1) / (16 * s.tiles));
    if (s.columns < 1) s.columns = 1;
    const int64_t keys = (int64_t)c->table_width * c->page_size < d->max_keys ? (int64_t)c->table_width * c->page_size : d->max_keys;
    const int64_t groups = (int64_t)c->batch * c->kv_heads * s.columns, least = 4 * KV4_TOKENS;
    const int64_t want = groups >= STEP_GROUPS ? 1 : STEP_GROUPS / groups;
    int64_t chunk = (keys + want - 1) / want;
    chunk = (chunk + least - 1) / least * least;
    if (chunk < least) chunk = least;
    s.waves = keys <= STEP_ALONE && chunk < keys ? 8 : 4;
    if (s.waves == 8) chunk = keys;
    s.splits = keys > 0 ? (int)((keys + chunk - 1) / chunk) : 1;
    s.chunk = (int)(s.splits == 1 ? 0x7fffffff / 512 * 512 : chunk);
    // (enough for any fewer tokens, which may be cut into more splits than these; where they have no splits fewer have none either)
    const int64_t most = want < (keys + least - 1) / least ? want : (keys + least - 1) / least;
    s.bytes = s.splits > 1 ? (size_t)most * d->rows * d->q_heads * (c->head_dim + 2) * 4 : 0;
    return s;
}

template <int DT, int D32, int T> void launch_step(const StepArgs& a, int waves, int batch, hipStream_t st) {
    const dim3 grid((unsigned)(a.splits * a.columns * a.heads), (unsigned)batch);
    if (waves == 8) hipLaunchKernelGGL((ogc_kv4_attention_kernel<DT, D32, T, 8>), grid, dim3(64 * 8), 0, st, a);
    else hipLaunchKernelGGL((ogc_kv4_attention_kernel<DT, D32, T, 4>), grid, dim3(64 * 4), 0, st, a);
}
template <int DT, int D32> void launch(const StepArgs& a, int waves, int tiles, int batch, hipStream_t st) {
    if constexpr (DT == OGC_BF16) {
        if (tiles == 2) launch_step<DT, D32, 2>(a, waves, batch, st);
        else launch_step<DT, D32, 1>(a, waves, batch, st);
    } else {
        launch_step<DT, D32, 1>(a, waves, batch, st);
    }
    if (a.splits > 1) {
        hipLaunchKernelGGL((ogc_kv4_attention_join_kernel<DT, D32 * 32>), dim3((unsigned)(a.max_rows * a.heads * a.group), (unsigned)batch), dim3(256), 0, st, a);
    }
}
template <int DT> void launch_dim(int d32, const StepArgs& a, int waves, int tiles, int batch, hipStream_t st) {
    switch (d32) {
    case 1: launch<DT, 1>(a, waves, tiles, batch, st); break;
    case 2: launch<DT, 2>(a, waves, tiles, batch, st); break;
    case 3: launch<DT, 3>(a, waves, tiles, batch, st); break;
    default: launch<DT, 4>(a, waves, tiles, batch, st); break;
    }
}

}  // namespace

extern "C" {

ogc_status ogc_kv4_attention_validate(const ogc_kv4_desc* c, const ogc_kv4_attention_desc* d) {
    if (!c || !d) return OGC_ERR_INVALID_ARG;
    if (d->dtype < OGC_F32 || d->dtype > OGC_F8) return OGC_ERR_INVALID_ARG;
    if (!(d->scale >= 0x1p-60f && d->scale <= 0x1p60f)) return OGC_ERR_INVALID_ARG;
    const ogc_status st = ogc_kv4_check(c);
    if (st != OGC_OK) return st;
    if (d->rows < 0 || d->max_rows < 0 || d->max_keys < 0 || d->q_heads <= 0) return OGC_ERR_SHAPE;
    if (d->q_heads % c->kv_heads != 0 || d->q_heads / c->kv_heads > 256) return OGC_ERR_SHAPE;
    const int max_rows = d->max_rows < d->rows ? d->max_rows : d->rows;
    if ((int64_t)max_rows * d->q_heads > 0x7fffff00) return OGC_ERR_SHAPE;
    if (d->dtype != OGC_F32 && d->dtype != OGC_BF16) return OGC_ERR_UNSUPPORTED;
    const StepShape s = shape_of(c, d);
    if ((int64_t)s.splits * s.columns * c->kv_heads * s.waves * 64 > 0xffffffff) return OGC_ERR_SHAPE;  // threads of a grid (a join's are far fewer)
    const int e = d->dtype == OGC_F32 ? 4 : 2;
    if (!strides_ok(d->q_stride, e) || !strides_ok(d->o_stride, e)) return OGC_ERR_ALIGNMENT;
    return OGC_OK;
}

ogc_status ogc_kv4_attention_workspace_bytes(const ogc_kv4_desc* c, const ogc_kv4_attention_desc* d, size_t* bytes) {
    const ogc_status st = ogc_kv4_attention_validate(c, d);
    if (st != OGC_OK) return st;
    if (!bytes) return OGC_ERR_INVALID_ARG;
    *bytes = shape_of(c, d).bytes;
    return OGC_OK;
}

ogc_status ogc_kv4_attention_run(const ogc_kv4_desc* c, const ogc_kv4_attention_desc* d, const void* q, const int32_t* cu,
                                 const int32_t* lens, const int32_t* page_table, const void* cache, void* o, void* workspace,
                                 void* stream) {
    const ogc_status st = ogc_kv4_attention_validate(c, d);
    if (st != OGC_OK) return st;
    if (d->rows == 0 || d->max_rows == 0) return OGC_OK;
    if (!q || !cu || !lens || !page_table || !cache || !o) return OGC_ERR_INVALID_ARG;
    if (((uintptr_t)q | (uintptr_t)cache | (uintptr_t)o | (uintptr_t)workspace) & 15) return OGC_ERR_ALIGNMENT;
    if (((uintptr_t)cu | (uintptr_t)lens | (uintptr_t)page_table) & 3) return OGC_ERR_ALIGNMENT;
    const StepShape s = shape_of(c, d);
    if (s.bytes > 0 && !workspace) return OGC_ERR_WORKSPACE;
    const int e = d->dtype == OGC_F32 ? 4 : 2;
    StepArgs a;
    a.q = (const uint8_t*)q;
    a.cache = (const uint8_t*)cache;
    a.o = (uint8_t*)o;
    a.cu = cu;
    a.lens = lens;
    a.table = page_table;
    a.partial = (float*)workspace;
    a.stats = s.splits > 1 ? (float*)workspace + (size_t)s.splits * d->rows * d->q_heads * c->head_dim : nullptr;
    for (int i = 0; i < 2; ++i) {
        a.sq[i] = d->q_stride[i] * e;
        a.so[i] = d->o_stride[i] * e;
    }
    a.rows = d->rows;
    a.max_rows = d->max_rows < d->rows ? d->max_rows : d->rows;
    const int64_t held = (int64_t)c->table_width * c->page_size;
    a.max_keys = (int)(held < d->max_keys ? held : d->max_keys);
    a.heads = c->kv_heads;
    a.group = d->q_heads / c->kv_heads;
    a.page_size = c->page_size;
    a.pages = c->pages;
    a.width = c->table_width;
    a.chunk = s.chunk;
    a.splits = s.splits;
    a.columns = s.columns;
    a.scale_log2 = d->scale * LOG2E;
    if (d->dtype == OGC_F32) launch_dim<OGC_F32>(c->head_dim / 32, a, s.waves, s.tiles, c->batch, (hipStream_t)stream);
    else launch_dim<OGC_BF16>(c->head_dim / 32, a, s.waves, s.tiles, c->batch, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? OGC_OK : OGC_ERR_DEVICE;
}

}  // extern "C"
