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
// scales from some 2^88 on they may overflow: a workgroup that finds a sum that is not finite starts again with a factor 2^-10.
// A scale of no number (byte 255) becomes an infinity here, and what is not finite then becomes NaN: values of the cache are finite
// otherwise, and so are their weighted means.
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

template <int N> struct Dwords;
template <> struct Dwords<1> { typedef uint32_t type; static __device__ __forceinline__ uint32_t at(type x, int) { return x; } };
template <> struct Dwords<2> { typedef v2u type; static __device__ __forceinline__ uint32_t at(const type& x, int i) { return x[i]; } };
template <> struct Dwords<3> { typedef v3u type; static __device__ __forceinline__ uint32_t at(const type& x, int i) { return x[i]; } };
template <> struct Dwords<4> { typedef v4u type; static __device__ __forceinline__ uint32_t at(const type& x, int i) { return x[i]; } };

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

template <int D32> struct Record {  // what a lane needs of a record
    static constexpr int NS = D32 == 3 ? 3 : 1;  // its channels have one scale, or (96 channels) up to three of them
    typename Dwords<D32>::type k[2];
    v2u v[D32], ks[NS], vs[D32];
    __device__ __forceinline__ void load(const uint8_t* r, int lane) {
        constexpr int D = D32 * 32;
        const int g = lane >> 4, m = lane & 15, t = 8 * (m / 4);
#pragma unroll
        for (int b = 0; b < 2; ++b) k[b] = *(const typename Dwords<D32>::type*)(r + kv4_key_at(D, t + 4 * b + m % 4, 8 * D32 * g));
#pragma unroll
        for (int s = 0; s < NS; ++s) ks[s] = *(const v2u*)(r + kv4_key_scale_at(D, (D32 * g + s) / 4, t));
#pragma unroll
        for (int c = 0; c < D32; ++c) {
            v[c] = *(const v2u*)(r + kv4_value_at(D, g, 32 * c + m));
            vs[c] = *(const v2u*)(r + kv4_value_scale_at(D, c, 8 * g));
        }
    }
};

// DT: of the queries.  T: column tiles of a wavefront.  W: wavefronts, which take the records of the split in turn.
template <int DT, int D32, int T, int W> __global__ __launch_bounds__(64 * W) void ogc_kv4_attention_kernel(StepArgs a) {
    constexpr int D = D32 * 32, E = DT == OGC_F32 ? 4 : 2, P = DT == OGC_F32 ? 3 : 1, ROW = D + 4;
    __shared__ float stat_lds[2][W][16 * T];
    __shared__ __attribute__((aligned(16))) float o_lds[W][16][ROW];
    const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.y;
    const uint32_t x = blockIdx.x;
    const int head = x % (uint32_t)a.heads, y = x / (uint32_t)a.heads, split = y / (uint32_t)a.columns, c0 = y % (uint32_t)a.columns * 16 * T;
    const StepSequence s = sequence_of(a, b);
    const int k0 = split * a.chunk;  // (the host holds splits * chunk below 2^31)
    if (c0 >= s.n * a.group || (split > 0 && k0 >= s.len)) return;
    const int k1 = min(s.len, k0 + a.chunk);
    const int32_t* const entries = a.table + (int64_t)b * a.width;

    // ---- queries: the second operand of the first product, in one or three bf16 pieces
    v8bf q[T][P][D32];
    int limit[T];  // the last token that this lane's column sees
    float ref[T], sum[T];
    v4f out[T][D32][2];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int c = c0 + 16 * t + col, i = c / (uint32_t)a.group;
        const bool on = i < s.n;
        limit[t] = on ? s.off + i : -1;
        const uint8_t* p = a.q + (long long)(s.row0 + (on ? i : 0)) * a.sq[0] + (long long)(head * a.group + c - i * a.group) * a.sq[1] + g * D32 * 8 * E;
#pragma unroll
        for (int d = 0; d < D32; ++d) {
            if constexpr (P == 1) {
                const v4i z = {0, 0, 0, 0};
                q[t][0][d] = __builtin_bit_cast(v8bf, on ? *(const v4i*)(p + d * 16) : z);
            } else {
                const v4f z = {0.0f, 0.0f, 0.0f, 0.0f};
                const Pieces8 r = split8(on ? *(const v4f*)(p + d * 32) : z, on ? *(const v4f*)(p + d * 32 + 16) : z);
#pragma unroll
                for (int i = 0; i < 3; ++i) q[t][i][d] = __builtin_bit_cast(v8bf, r.p[i]);
            }
        }
    }
    const int first_limit = s.off + c0 / (uint32_t)a.group;  // of the first column: the least

    // ---- the records of this wavefront, one ahead
    auto record_at = [&](int token) -> const uint8_t* {  // (wavefront-uniform)
        if (token >= k1) return nullptr;
        const int64_t at = kv4_record_at(entries, a.width, a.page_size, a.pages, a.heads, D, token, head);
        return at < 0 ? nullptr : a.cache + at;
    };
    float factor = 30.0f;  // of the weights, base-2 logarithm
again:
#pragma unroll
    for (int t = 0; t < T; ++t) {
        ref[t] = -INFINITY;
        sum[t] = 0.0f;
#pragma unroll
        for (int d = 0; d < D32; ++d) out[t][d][0] = out[t][d][1] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
    }
    Record<D32> next;
    const int first = k0 + wave * KV4_TOKENS;
    const uint8_t* r = record_at(first);
    if (r) next.load(r, lane);
    for (int token = first; token < k1; token += W * KV4_TOKENS) {
        const Record<D32> x = next;
        const bool here = r != nullptr;
        r = record_at(token + W * KV4_TOKENS);
        if (r) next.load(r, lane);
        if (!here) continue;
        const bool whole = token + KV4_TOKENS - 1 <= first_limit;

        v4f sc[T][2];
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) {
            v8bf k[D32];
#pragma unroll
            for (int d = 0; d < D32; ++d) {
                // (a lane's byte: token 8 (m / 4) + 4 tile + m % 4 of the eight in ks)
                const v2u& ks = x.ks[Record<D32>::NS == 1 ? 0 : d];
                const float scale = __builtin_bit_cast(float, (ks[tile] >> (8 * (col & 3)) & 255u) << 23);
                k[d] = operand(Dwords<D32>::at(x.k[tile], d), scale);
            }
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
        v8bf w[T][P][D32];
#pragma unroll
        for (int t = 0; t < T; ++t) {
            // ---- the eight scores of this lane: tokens 8 g + j, base-2 logarithm
            float e[8], cand = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                e[j] = sc[t][j >> 2][j & 3] * a.scale_log2;
                if (!whole && token + 8 * g + j > limit[t]) e[j] = -INFINITY;
                cand = fmaxf(cand, e[j]);
            }
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
            for (int j = 0; j < 8; ++j) e[j] = __builtin_amdgcn_exp2f(e[j] + off);
            if constexpr (P == 1) {  // rounded once; the sum takes what the second product multiplies
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const uint32_t pr = pack_bf16(e[j], e[j + 1]);
                    sum[t] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, pr), (v2bf){(__bf16)1.0f, (__bf16)1.0f}, sum[t], false);
                    e[j] = __builtin_bit_cast(float, pr << 16);
                    e[j + 1] = __builtin_bit_cast(float, pr & 0xffff0000u);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[t] += e[j];
            }
#pragma unroll
            for (int d = 0; d < D32; ++d) {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    f[j] = e[j] * exponent(x.vs[d], j);
                    if (!whole && token + 8 * g + j > limit[t]) f[j] = 0.0f;  // (whatever stands there)
                }
                if constexpr (P == 1) {
                    const v4i r = {(int)upper_halves(f[0], f[1]), (int)upper_halves(f[2], f[3]), (int)upper_halves(f[4], f[5]), (int)upper_halves(f[6], f[7])};
                    w[t][0][d] = __builtin_bit_cast(v8bf, r);
                } else {
                    const Pieces8 r = split8((v4f){f[0], f[1], f[2], f[3]}, (v4f){f[4], f[5], f[6], f[7]});
#pragma unroll
                    for (int p = 0; p < 3; ++p) w[t][p][d] = __builtin_bit_cast(v8bf, r.p[p]);
                }
            }
        }
#pragma unroll
        for (int d = 0; d < D32; ++d)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const v8bf v = operand(x.v[d][h], 1.0f);
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    if constexpr (P == 1) {
                        out[t][d][h] = mma(v, w[t][0][d], out[t][d][h]);
                    } else {  // a record's sum by itself, small products first
                        v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int p = 2; p >= 0; --p) acc = mma(v, w[t][p][d], acc);
                        out[t][d][h] += acc;
                    }
                }
            }
    }

    bool finite = true;
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int d = 0; d < D32; ++d)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) finite = finite && fabsf(out[t][d][h][e]) < INFINITY;
    if (__syncthreads_or(!finite) && factor > 0.0f) {
        factor = -10.0f;
        goto again;
    }

    // ---- the wavefronts' shares together
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
        for (int u = threadIdx.x; u < 16 * D / 4; u += 64 * W) {
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
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = total == 0.0f ? 0.0f : fabsf(r[e]) < INFINITY ? r[e] * inv : NAN;
            if (a.splits > 1) {  // the mean of the split, its reference and its sum without the factor
                const long long at = ((long long)split * a.rows + row) * (a.heads * a.group) + hd;
                *(v4f*)(a.partial + at * D + ch) = r;
                if (ch == 0) {
                    a.stats[2 * at] = top;
                    a.stats[2 * at + 1] = total * (factor > 0.0f ? 0x1p-30f : 0x1p10f);
                }
            } else {
                uint8_t* p = a.o + (long long)row * a.so[0] + (long long)hd * a.so[1] + ch * E;
                if constexpr (DT == OGC_F32) *(v4f*)p = r;
                else *(v2u*)p = (v2u){pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
            }
        }
        if (t + 1 < T) __syncthreads();
    }
}

// The splits of a query and head together: four channels a thread.
template <int DT, int D> __global__ __launch_bounds__(256) void ogc_kv4_attention_join_kernel(StepArgs a) {
    const StepSequence s = sequence_of(a, blockIdx.y);
    const uint32_t u = blockIdx.x * 256 + threadIdx.x, heads = a.heads * a.group;
    const int ch = u % (D / 4) * 4, hd = u / (D / 4) % heads, i = u / (D / 4) / heads;
    if (i >= s.n) return;
    const int n = (s.len + a.chunk - 1) / a.chunk;
    const long long at = (long long)(s.row0 + i) * heads + hd, step = (long long)a.rows * heads;
    float top = -INFINITY, total = 0.0f;
    for (int k = 0; k < n; ++k) top = fmaxf(top, a.stats[2 * (at + k * step)]);
    v4f r = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < n; ++k) {
        const float m = a.stats[2 * (at + k * step)], l = a.stats[2 * (at + k * step) + 1];
        const float h = m == -INFINITY ? 0.0f : half_power(m - top);
        total += m == -INFINITY ? l : l * h * h;
        r += *(const v4f*)(a.partial + (at + k * step) * D + ch) * (m == -INFINITY ? l : l * h) * (m == -INFINITY ? 1.0f : h);
    }
    if (total != 0.0f) r *= 1.0f / total;
    uint8_t* p = a.o + (s.row0 + i) * a.so[0] + hd * a.so[1] + ch * (DT == OGC_F32 ? 4 : 2);
    if constexpr (DT == OGC_F32) *(v4f*)p = r;
    else *(v2u*)p = (v2u){pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
}

bool strides_ok(const int64_t s[2], int elt) { return s[0] >= 0 && s[1] >= 0 && s[0] * elt % 16 == 0 && s[1] * elt % 16 == 0; }

constexpr int STEP_WAVES = 4;

struct StepShape {
    int tiles, columns, chunk, splits;
    size_t bytes;
};
// How a call is cut.  Columns: 16 or (bf16) 32 a workgroup.  Tokens: as many splits as give the chip some 2048 workgroups, of 128
// tokens at least, which is a record for each wavefront.
StepShape shape_of(const ogc_kv4_desc* c, const ogc_kv4_attention_desc* d) {
    StepShape s;
    const int group = d->q_heads / c->kv_heads;
    const int max_rows = d->max_rows < d->rows ? d->max_rows : d->rows;
    const int64_t columns = (int64_t)max_rows * group;
    s.tiles = d->dtype == OGC_BF16 && columns > 16 ? 2 : 1;
    s.columns = (int)((columns + 16 * s.tiles - 1) / (16 * s.tiles));
    if (s.columns < 1) s.columns = 1;
    const int64_t keys = (int64_t)c->table_width * c->page_size < d->max_keys ? (int64_t)c->table_width * c->page_size : d->max_keys;
    const int64_t groups = (int64_t)c->batch * c->kv_heads * s.columns, least = STEP_WAVES * KV4_TOKENS;
    const int64_t want = groups >= 2048 ? 1 : 2048 / groups;
    int64_t chunk = (keys + want - 1) / want;
    chunk = (chunk + least - 1) / least * least;
    if (chunk < least) chunk = least;
    s.splits = keys > 0 ? (int)((keys + chunk - 1) / chunk) : 1;
    s.chunk = (int)(s.splits == 1 ? 0x7fffffff / least * least : chunk);
    s.bytes = s.splits > 1 ? (size_t)s.splits * d->rows * d->q_heads * (c->head_dim + 2) * 4 : 0;
    return s;
}

template <int DT, int D32, int T> void launch_step(const StepArgs& a, int batch, hipStream_t st) {
    const dim3 grid((unsigned)(a.splits * a.columns * a.heads), (unsigned)batch);
    hipLaunchKernelGGL((ogc_kv4_attention_kernel<DT, D32, T, STEP_WAVES>), grid, dim3(64 * STEP_WAVES), 0, st, a);
}
template <int DT, int D32> void launch(const StepArgs& a, int tiles, int batch, hipStream_t st) {
    if constexpr (DT == OGC_BF16) {
        if (tiles == 2) launch_step<DT, D32, 2>(a, batch, st);
        else launch_step<DT, D32, 1>(a, batch, st);
    } else {
        launch_step<DT, D32, 1>(a, batch, st);
    }
    if (a.splits > 1) {
        const int64_t items = (int64_t)a.max_rows * a.heads * a.group * (D32 * 8);
        hipLaunchKernelGGL((ogc_kv4_attention_join_kernel<DT, D32 * 32>), dim3((unsigned)((items + 255) / 256), (unsigned)batch), dim3(256), 0, st, a);
    }
}
template <int DT> void launch_dim(int d32, const StepArgs& a, int tiles, int batch, hipStream_t st) {
    switch (d32) {
    case 1: launch<DT, 1>(a, tiles, batch, st); break;
    case 2: launch<DT, 2>(a, tiles, batch, st); break;
    case 3: launch<DT, 3>(a, tiles, batch, st); break;
    default: launch<DT, 4>(a, tiles, batch, st); break;
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
    if ((int64_t)max_rows * d->q_heads * (c->head_dim / 4) > 0x7fffff00) return OGC_ERR_SHAPE;  // (a launch's items of a sequence)
    if (d->dtype != OGC_F32 && d->dtype != OGC_BF16) return OGC_ERR_UNSUPPORTED;
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
    if ((int64_t)s.splits * s.columns * a.heads > 0x7fffffff) return OGC_ERR_SHAPE;
    if (d->dtype == OGC_F32) launch_dim<OGC_F32>(c->head_dim / 32, a, s.tiles, c->batch, (hipStream_t)stream);
    else launch_dim<OGC_BF16>(c->head_dim / 32, a, s.tiles, c->batch, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? OGC_OK : OGC_ERR_DEVICE;
}

}  // extern "C"
