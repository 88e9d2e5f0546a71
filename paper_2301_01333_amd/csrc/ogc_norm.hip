// The residual's addition with the root-mean-square norm (include/ogc_mx.h): rows in their own type or in a microscaled format.
//
// Rows are read once, kept in registers, and written twice (the sum and its norm): the kernel is bound by memory, or by its launch.  A
// lane holds N runs of eight channels.  In its own type a workgroup has one row; in a microscaled format it has eight, eight lanes of a
// wavefront each, because the codes of eight rows are 128 bytes side by side in the matrix, and a wavefront's four runs of a row
// are a block of 256 channels, whose four scales are one word.  Where that leaves compute units without work, or rows are long, it has two rows, 32 lanes
// each, whose runs are such a block.  Many short rows are eight of a workgroup in any type.  Rows that do not fit the registers (N = 0) are read a second
// time for the norm.
// 8192 x 4096 in bf16 with a residual: in its own type 49 us (268 MB, 5.5 TB/s), to 8 bits 57 (236 MB, 4.1: the reads of eight rows and the codes' 128 bytes
// cost what they save).  Squares in 64 bits cost nothing there (50 us each of inputs from memory, as with sums
// of eight in fp32), and 6 of 65 us for 3000 x 11000.  Many wavefronts with few runs each: eight runs a lane 56 and 63; tried for 8 bits and no better: rows read a kilobyte at
// a time and turned in LDS (62).
#include "ogc_mx_rows.h"

#include <math.h>

namespace {

struct NormArgs {
    const uint8_t* x;
    const uint8_t* residual;  // or NULL
    const float* weight;
    uint8_t* sum;
    uint8_t* y;  // rows, or codes
    uint8_t* scales;
    long long sx, sr, ss, sy;  // bytes
    int rows, channels, padded;
    float eps;
    double inv;  // 1 / channels
};

constexpr int NORM_WAVES = 16;

// ROWS: of a workgroup
template <int DT, int OUT, int ROWS, int N> __global__ __launch_bounds__(64 * NORM_WAVES) void ogc_norm_kernel(NormArgs a) {
    constexpr int E = MxEight<DT>::E, LANES = 64 / ROWS;  // lanes of a row in a wavefront
    constexpr int SPAN = ROWS == 8 ? MX_BLOCK : LANES * 8, RUNS = SPAN / (LANES * 8);  // channels and runs that a wavefront takes in turn
    __shared__ double part[NORM_WAVES][ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    // (eight rows: workgroup i runs on XCD i % 8, and the four workgroups of 32 rows of the matrix shall be one XCD's)
    const uint32_t group = ROWS == 8 ? blockIdx.x / 32 * 32 + blockIdx.x % 8 * 4 + blockIdx.x / 8 % 4 : blockIdx.x;
    const int64_t row = (int64_t)group * ROWS + lane / LANES;
    const int j = lane % LANES;
    const bool on = row < a.rows;
    const int64_t r = on ? row : 0;
    const uint8_t *const x = a.x + r * a.sx, *const res = a.residual ? a.residual + r * a.sr : nullptr;
    uint8_t* const sum = a.residual ? a.sum + r * a.ss : nullptr;
    const auto first = [&](int i) { return (i / RUNS * waves + wave) * SPAN + i % RUNS * LANES * 8 + j * 8; };  // channel of a lane's run i
    const int limit = OUT == OGC_NORM_SAME ? a.channels : a.padded;
    const int runs = (limit + SPAN * waves - 1) / (SPAN * waves) * RUNS;

    MxEight<DT> held[N > 0 ? N : 1];
    double square = 0.0;  // in 64 bits: squares of all numbers are some there, and the factor of a row is the rounded one, whatever its length
    const auto take = [&](MxEight<DT>& s, const MxEight<DT>& more, int c) {
        const int there = on ? a.channels - c : 0;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = res ? s.get(i) + more.get(i) : s.get(i);
        if (res) {
            s.set(v);  // (rounded: the norm is the norm of what the next layer adds to)
            if (there > 0) s.store(sum + (int64_t)c * E, there);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) square = __builtin_fma((double)s.get(i), (double)s.get(i), square);
    };
    if constexpr (N > 0) {
        MxEight<DT> more[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = first(i), there = on ? a.channels - c : 0;
            held[i].load(x + (int64_t)c * E, there);
            if (res) more[i].load(res + (int64_t)c * E, there);
            else more[i].clear();
        }
#pragma unroll
        for (int i = 0; i < N; ++i) take(held[i], more[i], first(i));
    } else {
        for (int i = 0; i < runs; ++i) {
            const int c = first(i), there = on ? a.channels - c : 0;
            MxEight<DT> s, more;
            s.load(x + (int64_t)c * E, there);
            if (res) more.load(res + (int64_t)c * E, there);
            else more.clear();
            take(s, more, c);
        }
    }
#pragma unroll
    for (int m = 1; m < LANES; m *= 2) square += __shfl_xor(square, m);
    if (waves > 1) {
        if (j == 0) part[wave][lane / LANES] = square;
        __syncthreads();
        square = 0.0;
        for (int w = 0; w < waves; ++w) square += part[w][lane / LANES];
    }
    // The factor of the largest rows is no normal fp32 number, and that of the smallest ones is beyond all of them: there a value takes a part of it first, a power of two, without rounding (or what is
    // lost is below the smallest result).
    const double root = __builtin_sqrt(square * a.inv + (double)a.eps);
    const float power = root > 0x1p100 ? 0x1p-64f : root < 0x1p-100 ? 0x1p64f : 1.0f;
    const float f = (float)(1.0 / (root * (double)power));

    const auto give = [&](const MxEight<DT>& s, int c, uint32_t& scales, int i) {
        const int there = on ? a.channels - c : 0;
        float v[8];
        if (there >= 8) {
            const mx_v4f w0 = *(const mx_v4f*)(a.weight + c), w1 = *(const mx_v4f*)(a.weight + c + 4);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = s.get(k) * power * f * (k < 4 ? w0[k % 4] : w1[k % 4]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = k < there ? s.get(k) * power * f * a.weight[c + k] : 0.0f;
        }
        if constexpr (OUT == OGC_NORM_SAME) {
            MxEight<DT> y;
            y.set(v);
            if (there > 0) y.store(a.y + r * a.sy + (int64_t)c * E, there);
        } else {
            constexpr int FORMAT = OUT == OGC_NORM_MX8 ? OGC_MX8 : OGC_MX4;
            uint32_t e;
            const mx_v2u code = mx_quantized<FORMAT>(v, e);
            if (on && c < a.padded) {
                uint8_t* const o = a.y + mx_code_at(FORMAT, a.padded, (int)row, c);
                if constexpr (FORMAT == OGC_MX8) *(mx_v2u*)o = code;
                else *(uint32_t*)o = code[0];
            }
            if constexpr (ROWS == 8) {
                scales = i % 4 ? scales | e << (i % 4 * 8) : e;
                if (on && c < a.padded && i % 4 == 3 && j % 4 == 0) *(uint32_t*)(a.scales + mx_scales_at(a.padded, (int)row, c / MX_BLOCK, j / 4)) = scales;
            } else {
                if (on && c < a.padded && j % 4 == 0) a.scales[mx_scales_at(a.padded, (int)row, c / MX_BLOCK, j / 4 % 2) + j / 8] = (uint8_t)e;
            }
        }
    };
    uint32_t scales = 0;
    if constexpr (N > 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) give(held[i], first(i), scales, i);
    } else {
        const uint8_t* const again = res ? sum : x;  // (a lane reads what it wrote itself)
        for (int i = 0; i < runs; ++i) {
            const int c = first(i);
            MxEight<DT> s;
            s.load(again + (int64_t)c * E, on ? a.channels - c : 0);
            give(s, c, scales, i);
        }
    }
}

// Wavefronts of a row: as many as hold it in two runs (of eight rows: four) of their lanes, or more, where rows are few.
template <int DT, int OUT, int ROWS> void launch(const NormArgs& a, hipStream_t st) {
    constexpr int LANES = 64 / ROWS, SPAN = ROWS == 8 ? MX_BLOCK : LANES * 8, RUNS = SPAN / (LANES * 8), MOST = ROWS == 8 ? 4 : 2;
    const unsigned grid = (unsigned)(ROWS == 8 ? ((int64_t)a.rows + 255) / 256 * 32 : ((int64_t)a.rows + ROWS - 1) / ROWS);
    const int turns = ((OUT == OGC_NORM_SAME ? a.channels : a.padded) + SPAN - 1) / SPAN;
    int waves = 1;
    while (waves < NORM_WAVES && turns > waves && (turns * RUNS > waves * MOST || (int64_t)grid * waves < 4096)) waves *= 2;
    const int runs = (turns + waves - 1) / waves * RUNS;
    const dim3 g(grid), t(64 * waves);
    if constexpr (RUNS == 1) {
        if (runs <= 2) {
            if (runs <= 1) hipLaunchKernelGGL((ogc_norm_kernel<DT, OUT, ROWS, 1>), g, t, 0, st, a);
            else hipLaunchKernelGGL((ogc_norm_kernel<DT, OUT, ROWS, 2>), g, t, 0, st, a);
            return;
        }
    }
    constexpr bool EIGHT = DT == OGC_BF16 && !(ROWS == 8 && OUT == OGC_NORM_SAME);  // (in fp32 they would not fit the registers)
    if (runs <= 4 || (ROWS == 8 && !EIGHT)) {
        hipLaunchKernelGGL((ogc_norm_kernel<DT, OUT, ROWS, 4>), g, t, 0, st, a);
        return;
    }
    if constexpr (EIGHT) {
        if (runs <= 8 || ROWS == 8) {
            hipLaunchKernelGGL((ogc_norm_kernel<DT, OUT, ROWS, 8>), g, t, 0, st, a);
            return;
        }
    }
    if constexpr (ROWS != 8) hipLaunchKernelGGL((ogc_norm_kernel<DT, OUT, ROWS, 0>), g, t, 0, st, a);  // (eight rows are taken where they fit: see below)
}
template <int DT> void launch(int out, const NormArgs& a, hipStream_t s) {
    // Two rows each or eight, us, of inputs from memory: bf16 to 8 bits 64 x 8192 5.7 / 12.5, 4097 x 4096 29.7 / 30.9, 5000 x 4096 35.5 / 34.1, 8192 x 4096 52.6 / 50.3, 32000 x
    // 4096 241 / 175; to 4 bits 5000 x 4096 30.4 / 32.6, 8192 x 4096 46.2 / 48.4, 32000 x 4096 179 / 161; fp32 to 8 bits 5000 x 4096 55.6 / 63.7, 8192 x 4096 98 / 102,
    // 32000 x 4096 384 / 341.  Rows that eight of a workgroup cannot hold in registers: bf16 3000 x 11000 45 / 65, fp32 3000 x 11000 106 / 137.
    const bool few = a.rows <= (DT == OGC_F32 || out == OGC_NORM_MX4 ? 8192 : 4096) || a.padded > (DT == OGC_F32 ? 4096 : 8192);
    // Many short rows, eight each or one: bf16 30000 x 100 10.0 / 23.0, 30000 x 256 11.7 / 14.7, 3000 x 100 6.2 / 5.2, 30000 x 512 19.1 / 20.2.
    const bool short_rows = a.rows >= 8192 && a.padded == MX_BLOCK;
    if (out == OGC_NORM_SAME) short_rows ? launch<DT, OGC_NORM_SAME, 8>(a, s) : launch<DT, OGC_NORM_SAME, 1>(a, s);
    else if (out == OGC_NORM_MX4) few ? launch<DT, OGC_NORM_MX4, 2>(a, s) : launch<DT, OGC_NORM_MX4, 8>(a, s);
    else few ? launch<DT, OGC_NORM_MX8, 2>(a, s) : launch<DT, OGC_NORM_MX8, 8>(a, s);
}

bool aligned(int64_t stride, int e) { return stride >= 0 && stride * e % 16 == 0; }

}  // namespace

extern "C" {

ogc_status ogc_norm_validate(const ogc_norm_desc* d) {
    if (!d) return OGC_ERR_INVALID_ARG;
    if (d->dtype < OGC_F32 || d->dtype > OGC_F8 || d->out < OGC_NORM_SAME || d->out > OGC_NORM_MX8) return OGC_ERR_INVALID_ARG;
    if (!(d->eps >= 0.0f && isfinite(d->eps))) return OGC_ERR_INVALID_ARG;
    if (d->rows < 0 || d->channels <= 0 || d->channels > 1 << 20) return OGC_ERR_SHAPE;
    if (d->rows > 0x3fffff) return OGC_ERR_SHAPE;  // a workgroup of up to 1024 threads for each: a grid of fewer than 2^32
    if (d->dtype != OGC_F32 && d->dtype != OGC_BF16) return OGC_ERR_UNSUPPORTED;
    const int e = d->dtype == OGC_F32 ? 4 : 2;
    if (!aligned(d->x_stride, e) || !aligned(d->residual_stride, e) || !aligned(d->sum_stride, e)) return OGC_ERR_ALIGNMENT;
    if (d->out == OGC_NORM_SAME && !aligned(d->y_stride, e)) return OGC_ERR_ALIGNMENT;
    return OGC_OK;
}

ogc_status ogc_norm_run(const ogc_norm_desc* d, const void* x, const void* residual, const float* weight, void* sum, void* y,
                        void* scales, void* stream) {
    const ogc_status st = ogc_norm_validate(d);
    if (st != OGC_OK) return st;
    if (d->rows == 0) return OGC_OK;
    const bool same = d->out == OGC_NORM_SAME;
    if (!x || !weight || !y || (residual && !sum) || (!same && !scales)) return OGC_ERR_INVALID_ARG;
    if (((uintptr_t)x | (uintptr_t)weight | (uintptr_t)y) & 15) return OGC_ERR_ALIGNMENT;
    if (residual && (((uintptr_t)residual | (uintptr_t)sum) & 15)) return OGC_ERR_ALIGNMENT;
    if (!same && ((uintptr_t)scales & 15)) return OGC_ERR_ALIGNMENT;
    const int e = d->dtype == OGC_F32 ? 4 : 2;
    NormArgs a;
    a.x = (const uint8_t*)x;
    a.residual = (const uint8_t*)residual;
    a.weight = weight;
    a.sum = (uint8_t*)sum;
    a.y = (uint8_t*)y;
    a.scales = (uint8_t*)scales;
    a.sx = d->x_stride * e;
    a.sr = d->residual_stride * e;
    a.ss = d->sum_stride * e;
    a.sy = d->y_stride * e;
    a.rows = d->rows;
    a.channels = d->channels;
    a.padded = mx_padded_channels(d->channels);
    a.eps = d->eps;
    a.inv = 1.0 / (double)d->channels;
    const hipStream_t s = (hipStream_t)stream;
    if (d->dtype == OGC_F32) launch<OGC_F32>(d->out, a, s);
    else launch<OGC_BF16>(d->out, a, s);
    return hipGetLastError() == hipSuccess ? OGC_OK : OGC_ERR_DEVICE;
}

}  // extern "C"
