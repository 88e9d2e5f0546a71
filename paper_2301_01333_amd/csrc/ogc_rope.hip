// Norms of queries and keys for each head, with the rotation of their positions in the same pass (include/ogc_decoder.h).
//
// Every value is read and written once and meets a few instructions: the kernel is bound by memory, and by its launch where
// rows are few.  A lane owns two runs of VC channels of a row, chosen so that both members of every pair are its own (HALF: run s and the
// run rot/2 further; INTERLEAVED: two neighbouring runs) and that both layouts turn by the same angles s * VC ..: nothing
// crosses lanes but the sum of squares.  The angles of a token are the same for all its heads: one wavefront computes them once, an
// angle a lane, and its lanes take theirs from LDS for all the heads that it covers.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "ogc_decoder.h"

namespace {

struct RopeArgs {
    const uint8_t* q;
    const uint8_t* k;
    const float* qw;
    const float* kw;
    const int32_t* pos;
    const double* freq;
    uint8_t* qo;
    uint8_t* ko;
    long long sq[2], sk[2], sqo[2], sko[2];  // bytes: row, head
    int tokens, q_heads, heads;              // heads: of queries and keys together
    int rot, interleaved, norm;
    int parts, passes;  // wavefronts of a token, rows a lane group takes one after the other
    float eps, magnitude;
};

typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

// VC values of a row in memory as fp32 and back (bf16: rounded to nearest even)
template <int DT, int VC> struct Run;
template <> struct Run<OGC_F32, 4> {
    v4f raw;
    __device__ __forceinline__ void load(const uint8_t* p) { raw = *(const v4f*)p; }
    __device__ __forceinline__ void get(float (&x)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = raw[i];
    }
    static __device__ __forceinline__ void store(uint8_t* p, const float (&x)[4]) { *(v4f*)p = (v4f){x[0], x[1], x[2], x[3]}; }
};
template <int VC> struct Run<OGC_BF16, VC> {
    typedef uint32_t vec __attribute__((ext_vector_type(VC / 2)));
    vec raw;
    __device__ __forceinline__ void load(const uint8_t* p) { raw = *(const vec*)p; }
    __device__ __forceinline__ void get(float (&x)[VC]) const {
#pragma unroll
        for (int i = 0; i < VC / 2; ++i) {
            const uint32_t w = raw[i];
            x[2 * i] = __builtin_bit_cast(float, w << 16);
            x[2 * i + 1] = __builtin_bit_cast(float, w & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void store(uint8_t* p, const float (&x)[VC]) {
        vec r;
#pragma unroll
        for (int i = 0; i < VC / 2; ++i) {
            const v2bf t = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
            r[i] = __builtin_bit_cast(uint32_t, t);
        }
        *(vec*)p = r;
    }
};

// cosine and sine of position * frequency.  The product and its reduction by quarter turns are in 64 bits (a quarter turn is taken off in two
// pieces: 2^31 of them leave 2^-50 of error), the two series on [-pi/4, pi/4] as well: their first terms left out are
// below 7e-12 and 3.9e-13, so that the result is the rounded one but for ties.  One lane does it for all heads of a token.
__device__ __forceinline__ v2f turn_of(int position, double frequency, float magnitude) {
    const double angle = (double)position * frequency;
    const double quarters = __builtin_rint(angle * 0.63661977236758134308);
    double r = __builtin_fma(-quarters, 1.57079632679489655800, angle);
    r = __builtin_fma(-quarters, 6.12323399573676603587e-17, r);
    const double x = r * r;
    const double s = r + r * x * (-1.0 / 6 + x * (1.0 / 120 + x * (-1.0 / 5040 + x * (1.0 / 362880 + x * (-1.0 / 39916800)))));
    const double c = 1.0 + x * (-0.5 + x * (1.0 / 24 + x * (-1.0 / 720 + x * (1.0 / 40320 + x * (-1.0 / 3628800 + x * (1.0 / 479001600))))));
    const long long n = (long long)quarters;
    const double cs = n & 1 ? s : c, sn = n & 1 ? c : s;
    const bool finite = __builtin_fabs(angle) < 0x1p62;  // (an angle that is no number turns into none)
    v2f t;
    t[0] = finite ? (float)((n + 1) & 2 ? -cs : cs) * magnitude : NAN;
    t[1] = finite ? (float)(n & 2 ? -sn : sn) * magnitude : NAN;
    return t;
}

template <int DT, int VC, int D> __global__ __launch_bounds__(256) void ogc_rope_kernel(RopeArgs a) {
    constexpr int E = DT == OGC_F32 ? 4 : 2;
    constexpr int SLOTS = D / (2 * VC), L = SLOTS <= 2 ? 2 : SLOTS <= 4 ? 4 : SLOTS <= 8 ? 8 : 16, ROWS = 64 / L;  // lanes and rows of a wavefront
    __shared__ v2f turns[4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t w = blockIdx.x * 4 + wave;  // (fits: checked by the host)
    const int token = w / (uint32_t)a.parts, part = w % (uint32_t)a.parts;
    const bool on = token < a.tokens;
    const int slot = lane % L, rows0 = part * a.passes * ROWS + lane / L;
    const bool turned = slot * 2 * VC < a.rot;
    const int c0 = turned && !a.interleaved ? slot * VC : slot * 2 * VC;
    const int c1 = turned && !a.interleaved ? a.rot / 2 + slot * VC : slot * 2 * VC + VC;
    const bool mine = on && (SLOTS == L || slot < SLOTS);

    if (on && lane < a.rot / 2) turns[wave][lane] = turn_of(a.pos[token], a.freq[lane], a.magnitude);
    __syncthreads();
    float cs[VC], sn[VC];
#pragma unroll
    for (int j = 0; j < VC; ++j) {
        const v2f t = turned ? turns[wave][slot * VC + j] : (v2f){1.0f, 0.0f};
        cs[j] = t[0], sn[j] = t[1];
    }
    for (int i = 0; i < a.passes; ++i) {
        const int row = rows0 + i * ROWS;
        const bool there = mine && row < a.heads, is_k = row >= a.q_heads;
        const int head = is_k ? row - a.q_heads : row;
        float x0[VC], x1[VC];
#pragma unroll
        for (int j = 0; j < VC; ++j) x0[j] = x1[j] = 0.0f;
        if (there) {
            const uint8_t* p = is_k ? a.k + token * a.sk[0] + head * a.sk[1] : a.q + token * a.sq[0] + head * a.sq[1];
            Run<DT, VC> u, v;
            u.load(p + c0 * E);
            v.load(p + c1 * E);
            u.get(x0);
            v.get(x1);
        }
        if (a.norm) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < VC; ++j) sum = __builtin_fmaf(x0[j], x0[j], __builtin_fmaf(x1[j], x1[j], sum));
#pragma unroll
            for (int m = 1; m < L; m *= 2) sum += __shfl_xor(sum, m);
            const float f = rsqrtf(sum * (1.0f / D) + a.eps);
            if (there) {
                const float* wt = is_k ? a.kw : a.qw;
#pragma unroll
                for (int j = 0; j < VC; j += 4) {
                    const v4f w0 = *(const v4f*)(wt + c0 + j), w1 = *(const v4f*)(wt + c1 + j);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x0[j + e] = x0[j + e] * f * w0[e];
                        x1[j + e] = x1[j + e] * f * w1[e];
                    }
                }
            }
        }
        if (!there) continue;
        float y0[VC], y1[VC];
        if (!turned) {
#pragma unroll
            for (int j = 0; j < VC; ++j) y0[j] = x0[j], y1[j] = x1[j];
        } else if (!a.interleaved) {
#pragma unroll
            for (int j = 0; j < VC; ++j) {
                y0[j] = x0[j] * cs[j] - x1[j] * sn[j];
                y1[j] = x0[j] * sn[j] + x1[j] * cs[j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < VC / 2; ++j) {
                y0[2 * j] = x0[2 * j] * cs[j] - x0[2 * j + 1] * sn[j];
                y0[2 * j + 1] = x0[2 * j] * sn[j] + x0[2 * j + 1] * cs[j];
                y1[2 * j] = x1[2 * j] * cs[VC / 2 + j] - x1[2 * j + 1] * sn[VC / 2 + j];
                y1[2 * j + 1] = x1[2 * j] * sn[VC / 2 + j] + x1[2 * j + 1] * cs[VC / 2 + j];
            }
        }
        uint8_t* o = is_k ? a.ko + token * a.sko[0] + head * a.sko[1] : a.qo + token * a.sqo[0] + head * a.sqo[1];
        Run<DT, VC>::store(o + c0 * E, y0);
        Run<DT, VC>::store(o + c1 * E, y1);
    }
}

bool strides_ok(const int64_t s[2], int elt) { return s[0] >= 0 && s[1] >= 0 && s[0] * elt % 16 == 0 && s[1] * elt % 16 == 0; }

template <int DT, int VC> void launch(int d, const RopeArgs& a, unsigned grid, hipStream_t st) {
    switch (d) {
    case 32: hipLaunchKernelGGL((ogc_rope_kernel<DT, VC, 32>), dim3(grid), dim3(256), 0, st, a); break;
    case 64: hipLaunchKernelGGL((ogc_rope_kernel<DT, VC, 64>), dim3(grid), dim3(256), 0, st, a); break;
    case 96: hipLaunchKernelGGL((ogc_rope_kernel<DT, VC, 96>), dim3(grid), dim3(256), 0, st, a); break;
    default: hipLaunchKernelGGL((ogc_rope_kernel<DT, VC, 128>), dim3(grid), dim3(256), 0, st, a); break;
    }
}

}  // namespace

extern "C" {

ogc_status ogc_rope_validate(const ogc_rope_desc* d) {
    if (!d) return OGC_ERR_INVALID_ARG;
    if (d->dtype < OGC_F32 || d->dtype > OGC_F8) return OGC_ERR_INVALID_ARG;
    if (d->layout != OGC_ROPE_HALF && d->layout != OGC_ROPE_INTERLEAVED) return OGC_ERR_INVALID_ARG;
    if (d->norm != 0 && d->norm != 1) return OGC_ERR_INVALID_ARG;
    if (d->norm && !(d->eps >= 0.0f && isfinite(d->eps))) return OGC_ERR_INVALID_ARG;
    if (!isfinite(d->magnitude)) return OGC_ERR_INVALID_ARG;
    if (d->tokens < 0 || d->q_heads <= 0 || d->kv_heads <= 0 || d->head_dim <= 0 || d->rot_dim < 0 || d->rot_dim > d->head_dim) return OGC_ERR_SHAPE;
    if (d->q_heads > 65536 || d->kv_heads > 65536) return OGC_ERR_SHAPE;
    if (d->tokens > 4 * 0xffffff) return OGC_ERR_SHAPE;  // four a workgroup (but where they are few), and a grid of fewer than 2^32 threads
    if (d->dtype != OGC_F32 && d->dtype != OGC_BF16) return OGC_ERR_UNSUPPORTED;
    if (d->head_dim % 32 != 0 || d->head_dim > 128 || d->rot_dim % 8 != 0) return OGC_ERR_UNSUPPORTED;
    const int e = d->dtype == OGC_F32 ? 4 : 2;
    if (!strides_ok(d->q_stride, e) || !strides_ok(d->k_stride, e) || !strides_ok(d->qo_stride, e) || !strides_ok(d->ko_stride, e))
        return OGC_ERR_ALIGNMENT;
    return OGC_OK;
}

ogc_status ogc_rope_run(const ogc_rope_desc* d, const void* q, const void* k, const float* q_weight, const float* k_weight,
                        const int32_t* positions, const double* frequencies, void* q_out, void* k_out, void* stream) {
    const ogc_status st = ogc_rope_validate(d);
    if (st != OGC_OK) return st;
    if (d->tokens == 0) return OGC_OK;
    if (!q || !k || !q_out || !k_out) return OGC_ERR_INVALID_ARG;
    if (d->norm && (!q_weight || !k_weight)) return OGC_ERR_INVALID_ARG;
    if (d->rot_dim && (!positions || !frequencies)) return OGC_ERR_INVALID_ARG;
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)q_out | (uintptr_t)k_out) & 15) return OGC_ERR_ALIGNMENT;
    if (d->norm && (((uintptr_t)q_weight | (uintptr_t)k_weight) & 15)) return OGC_ERR_ALIGNMENT;
    if (d->rot_dim && (((uintptr_t)positions & 3) || ((uintptr_t)frequencies & 7))) return OGC_ERR_ALIGNMENT;
    const int e = d->dtype == OGC_F32 ? 4 : 2;
    RopeArgs a;
    a.q = (const uint8_t*)q;
    a.k = (const uint8_t*)k;
    a.qw = q_weight;
    a.kw = k_weight;
    a.pos = positions;
    a.freq = frequencies;
    a.qo = (uint8_t*)q_out;
    a.ko = (uint8_t*)k_out;
    for (int i = 0; i < 2; ++i) {
        a.sq[i] = d->q_stride[i] * e;
        a.sk[i] = d->k_stride[i] * e;
        a.sqo[i] = d->qo_stride[i] * e;
        a.sko[i] = d->ko_stride[i] * e;
    }
    a.tokens = d->tokens;
    a.q_heads = d->q_heads;
    a.heads = d->q_heads + d->kv_heads;
    a.rot = d->rot_dim;
    a.interleaved = d->layout == OGC_ROPE_INTERLEAVED;
    a.norm = d->norm;
    a.eps = d->eps;
    a.magnitude = d->magnitude;
    // Runs of 16 bytes where a half of the rotated channels is a whole number of them, else (bf16) of 8.
    const bool wide = d->dtype == OGC_F32 || d->rot_dim % 16 == 0;
    const int vc = d->dtype == OGC_F32 || !wide ? 4 : 8;
    int lanes = 2;
    while (lanes < d->head_dim / (2 * vc)) lanes *= 2;
    const int rows = 64 / lanes, rounds = (a.heads + rows - 1) / rows;
    // A wavefront takes all heads of a token, unless that leaves the chip without work: then they are shared.
    a.parts = 1;
    while (a.parts < rounds && (int64_t)d->tokens * a.parts < 4096) ++a.parts;
    a.passes = (rounds + a.parts - 1) / a.parts;
    a.parts = (rounds + a.passes - 1) / a.passes;
    const int64_t grid = ((int64_t)d->tokens * a.parts + 3) / 4;  // (below 2^24: more than one wavefront a token only where they are few)
    const hipStream_t s = (hipStream_t)stream;
    if (d->dtype == OGC_F32) launch<OGC_F32, 4>(d->head_dim, a, (unsigned)grid, s);
    else if (wide) launch<OGC_BF16, 8>(d->head_dim, a, (unsigned)grid, s);
    else launch<OGC_BF16, 4>(d->head_dim, a, (unsigned)grid, s);
    return hipGetLastError() == hipSuccess ? OGC_OK : OGC_ERR_DEVICE;
}

}  // extern "C"
