// Rows in microscaled formats: written and read back (include/ogc_mx.h; their product: ogc_mx_product.hip).
//
// Both kernels move every value once and are bound by memory, or by their launch.  A workgroup has 256 channels of 32 rows, a wavefront eight
// of the rows, a lane eight channels of each of four runs of 64: rows are read 128 bytes (fp32: 256) at a time, the codes
// of eight rows leave as 128 bytes side by side, and a lane's four scales of a row are one word of the matrix.  bf16, 4096 x 8192: a gated pair to 8 bits 36 us
// (169 MB, 4.7 TB/s), back 16 us (101 MB, 6.2 TB/s); fp32, 2001 x 4500: to 4 bits 8.6 us (41 MB, 4.8 TB/s).
#include "ogc_mx_rows.h"

#include <math.h>

namespace {

struct RowsArgs {
    uint8_t* x;  // rows: read by the writing kernel, written by the reading one
    uint8_t* codes;
    uint8_t* scales;
    long long stride;  // bytes
    int rows, channels, padded, blocks;  // blocks: of 256 channels
};

// a * b / (1 + exp(-a)) for a from -80 on, but 0 < |a| < 2^-125: there neither exp(-|a|) nor its product with a is below the normal numbers, which the instruction for powers of two does not give,
// and only the last product is rounded to what is there.  exp(-|a|) does not lose what the product of |a| and log2(e) is rounded by (and is 0 from some 87 on).
MX_DEV float gated(float a, float b) {
    const float m = __builtin_fmaxf(-__builtin_fabsf(a), -128.0f), hi = m * 1.44269502162933349609f;
    const float lo = __builtin_fmaf(m, 1.44269502162933349609f, -hi) + m * 1.92596299112661746887e-8f;
    float t = __builtin_amdgcn_exp2f(hi);
    t = __builtin_fmaf(t, lo * 0.69314718055994530942f, t);
    return a * ((a < 0.0f ? t : 1.0f) * __builtin_amdgcn_rcpf(1.0f + t)) * b;  // (the reciprocal is off by 2^-23)
}
// The same for every a, in 64 bits: b may be as large as exp(-|a|) is small.  (e^-512 of any two numbers is none.)
MX_DEV float gated_far(float a, float b) {
    const float m = __builtin_fmaxf(-__builtin_fabsf(a), -512.0f), hi = m * 1.44269502162933349609f, n = __builtin_rintf(hi);
    const float lo = __builtin_fmaf(m, 1.44269502162933349609f, -hi) + m * 1.92596299112661746887e-8f;
    const float f = __builtin_amdgcn_exp2f(hi - n);
    const double t = __builtin_amdgcn_ldexp((double)__builtin_fmaf(f, lo * 0.69314718055994530942f, f), (int)n);
    return (float)((double)a * (a < 0.0f ? t : 1.0) / (1.0 + t) * (double)b);
}

template <int DT, int FORMAT, int GATE> __global__ __launch_bounds__(256) void ogc_mx_write_kernel(RowsArgs a) {
    constexpr int E = MxEight<DT>::E;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = blockIdx.x % (uint32_t)a.blocks;
    const int64_t row = (int64_t)(blockIdx.x / (uint32_t)a.blocks) * MX_ROWS + wave * 8 + lane / 8;
    const int j = lane % 8, c0 = block * MX_BLOCK + j * 8;
    const bool on = row < a.rows;
    const uint8_t* const p = a.x + (on ? row : 0) * a.stride;
    MxEight<DT> x[4], y[GATE ? 4 : 1];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const int c = c0 + s * 64, there = on ? a.channels - c : 0;
        x[s].load(p + (int64_t)c * E, there);
        if constexpr (GATE) y[s].load(p + ((int64_t)a.channels + c) * E, there);  // (of any alignment of a channel)
    }
    uint32_t scales = 0;
    mx_v2u code[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = GATE ? gated(x[s].get(i), y[GATE ? s : 0].get(i)) : x[s].get(i);
        if constexpr (GATE) {
            // (of the bits: negative numbers are above the others, and the larger the further from 0)
            uint32_t most = 0, nearest = 0xffffffffu;  // nearest to 0, which is none itself
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t bits = __builtin_bit_cast(uint32_t, x[s].get(i));
                most = max(most, bits);
                if constexpr (DT == OGC_F32) nearest = min(nearest, (bits & 0x7fffffffu) - 1);  // (bf16: a half of the smallest is a number of fp32)
            }
            const bool far = (most > 0xc2a00000u) | (nearest < 0x00ffffffu);  // -80; 2^-125 is 0x01000000
            if (__builtin_expect(far, 0)) {
                MxEight<DT> p = x[s], q = y[GATE ? s : 0];
#pragma unroll 1
                for (int i = 0; i < 8; ++i) {  // (a loop, of a value at a time: code that is hardly ever run shall not be in the way of the other)
                    const float far_one = gated_far(p.get(0), q.get(0));
#pragma unroll
                    for (int k = 0; k < 7; ++k) v[k] = v[k + 1];
                    v[7] = far_one;
                    p.next();
                    q.next();
                }
            }
        }
        uint32_t e;
        code[s] = mx_quantized<FORMAT>(v, e);
        scales |= e << (8 * s);
    }
    if (!on) return;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        uint8_t* const o = a.codes + mx_code_at(FORMAT, a.padded, (int)row, c0 + s * 64);
        if constexpr (FORMAT == OGC_MX8) *(mx_v2u*)o = code[s];
        else *(uint32_t*)o = code[s][0];
    }
    if (j % 4 == 0) *(uint32_t*)(a.scales + mx_scales_at(a.padded, (int)row, block, j / 4)) = scales;
}

template <int DT, int FORMAT> __global__ __launch_bounds__(256) void ogc_mx_read_kernel(RowsArgs a) {
    constexpr int E = MxEight<DT>::E;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = blockIdx.x % (uint32_t)a.blocks;
    const int64_t row = (int64_t)(blockIdx.x / (uint32_t)a.blocks) * MX_ROWS + wave * 8 + lane / 8;
    const int j = lane % 8, c0 = block * MX_BLOCK + j * 8;
    if (row >= a.rows) return;
    const uint32_t scales = *(const uint32_t*)(a.scales + mx_scales_at(a.padded, (int)row, block, j / 4));
    mx_v2u code[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const uint8_t* const o = a.codes + mx_code_at(FORMAT, a.padded, (int)row, c0 + s * 64);
        if constexpr (FORMAT == OGC_MX8) code[s] = *(const mx_v2u*)o;
        else code[s] = (mx_v2u){*(const uint32_t*)o, 0};
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const uint32_t e = scales >> (8 * s) & 255;
        const float scale = __builtin_bit_cast(float, e << 23);
        float v[8];
        if constexpr (FORMAT == OGC_MX4) {
            mx_v2f t[4];
            t[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[s][0], scale, 0);
            t[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[s][0], scale, 1);
            t[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[s][0], scale, 2);
            t[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[s][0], scale, 3);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = t[i / 2][i % 2];
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const mx_v2f t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code[s][h], scale, false);
                const mx_v2f u = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code[s][h], scale, true);
                v[4 * h] = t[0], v[4 * h + 1] = t[1], v[4 * h + 2] = u[0], v[4 * h + 3] = u[1];
            }
        }
        const int c = c0 + s * 64;
        if (c >= a.channels) break;
        MxEight<DT> y;
        y.set(v);
        y.store(a.x + row * a.stride + (int64_t)c * E, a.channels - c);
    }
}

template <bool WRITE> ogc_status move(const ogc_mx_rows* d, const void* x, const void* codes, const void* scales, void* stream) {
    const ogc_status st = ogc_mx_validate(d);
    if (st != OGC_OK) return st;
    if (!WRITE && d->gate != OGC_GATE_NONE) return OGC_ERR_INVALID_ARG;
    if (d->rows == 0) return OGC_OK;
    if (!x || !codes || !scales) return OGC_ERR_INVALID_ARG;
    if (((uintptr_t)x | (uintptr_t)codes | (uintptr_t)scales) & 15) return OGC_ERR_ALIGNMENT;
    const int e = d->dtype == OGC_F32 ? 4 : 2;
    RowsArgs a;
    a.x = (uint8_t*)const_cast<void*>(x);
    a.codes = (uint8_t*)const_cast<void*>(codes);
    a.scales = (uint8_t*)const_cast<void*>(scales);
    a.stride = d->stride * e;
    a.rows = d->rows;
    a.channels = d->channels;
    a.padded = mx_padded_channels(d->channels);
    a.blocks = a.padded / MX_BLOCK;
    const dim3 grid((unsigned)(mx_padded_rows(d->rows) / MX_ROWS * a.blocks)), threads(256);  // (checked: below 2^24)
    const hipStream_t s = (hipStream_t)stream;
    const int which = (d->dtype == OGC_F32 ? 4 : 0) + (d->format == OGC_MX8 ? 2 : 0) + (d->gate == OGC_GATE_SILU ? 1 : 0);
    if constexpr (WRITE) {
        switch (which) {
        case 0: hipLaunchKernelGGL((ogc_mx_write_kernel<OGC_BF16, OGC_MX4, 0>), grid, threads, 0, s, a); break;
        case 1: hipLaunchKernelGGL((ogc_mx_write_kernel<OGC_BF16, OGC_MX4, 1>), grid, threads, 0, s, a); break;
        case 2: hipLaunchKernelGGL((ogc_mx_write_kernel<OGC_BF16, OGC_MX8, 0>), grid, threads, 0, s, a); break;
        case 3: hipLaunchKernelGGL((ogc_mx_write_kernel<OGC_BF16, OGC_MX8, 1>), grid, threads, 0, s, a); break;
        case 4: hipLaunchKernelGGL((ogc_mx_write_kernel<OGC_F32, OGC_MX4, 0>), grid, threads, 0, s, a); break;
        case 5: hipLaunchKernelGGL((ogc_mx_write_kernel<OGC_F32, OGC_MX4, 1>), grid, threads, 0, s, a); break;
        case 6: hipLaunchKernelGGL((ogc_mx_write_kernel<OGC_F32, OGC_MX8, 0>), grid, threads, 0, s, a); break;
        default: hipLaunchKernelGGL((ogc_mx_write_kernel<OGC_F32, OGC_MX8, 1>), grid, threads, 0, s, a); break;
        }
    } else {
        switch (which) {
        case 0: hipLaunchKernelGGL((ogc_mx_read_kernel<OGC_BF16, OGC_MX4>), grid, threads, 0, s, a); break;
        case 2: hipLaunchKernelGGL((ogc_mx_read_kernel<OGC_BF16, OGC_MX8>), grid, threads, 0, s, a); break;
        case 4: hipLaunchKernelGGL((ogc_mx_read_kernel<OGC_F32, OGC_MX4>), grid, threads, 0, s, a); break;
        default: hipLaunchKernelGGL((ogc_mx_read_kernel<OGC_F32, OGC_MX8>), grid, threads, 0, s, a); break;
        }
    }
    return hipGetLastError() == hipSuccess ? OGC_OK : OGC_ERR_DEVICE;
}

}  // namespace

extern "C" {

ogc_status ogc_mx_bytes(int32_t format, int32_t rows, int32_t channels, size_t* codes, size_t* scales) {
    if (!codes || !scales || (format != OGC_MX4 && format != OGC_MX8)) return OGC_ERR_INVALID_ARG;
    if (rows < 0 || channels <= 0 || channels > 1 << 20) return OGC_ERR_SHAPE;
    const int padded = mx_padded_channels(channels);
    *codes = (size_t)(mx_padded_rows(rows) / MX_ROWS * mx_codes_of_32(format, padded));
    *scales = (size_t)(mx_padded_rows(rows) / MX_ROWS * padded);
    return OGC_OK;
}

ogc_status ogc_mx_validate(const ogc_mx_rows* d) {
    if (!d) return OGC_ERR_INVALID_ARG;
    if (d->dtype < OGC_F32 || d->dtype > OGC_F8 || (d->format != OGC_MX4 && d->format != OGC_MX8)) return OGC_ERR_INVALID_ARG;
    if (d->gate != OGC_GATE_NONE && d->gate != OGC_GATE_SILU) return OGC_ERR_INVALID_ARG;
    if (d->rows < 0 || d->channels <= 0 || d->channels > 1 << 20) return OGC_ERR_SHAPE;
    if (mx_padded_rows(d->rows) / MX_ROWS * (mx_padded_channels(d->channels) / MX_BLOCK) > 0xffffff) return OGC_ERR_SHAPE;  // a grid of fewer than 2^32 threads
    if (d->dtype != OGC_F32 && d->dtype != OGC_BF16) return OGC_ERR_UNSUPPORTED;
    if (d->stride < 0 || d->stride * (d->dtype == OGC_F32 ? 4 : 2) % 16 != 0) return OGC_ERR_ALIGNMENT;
    return OGC_OK;
}

ogc_status ogc_mx_write(const ogc_mx_rows* d, const void* x, void* codes, void* scales, void* stream) {
    return move<true>(d, x, codes, scales, stream);
}

ogc_status ogc_mx_read(const ogc_mx_rows* d, const void* codes, const void* scales, void* y, void* stream) {
    return move<false>(d, y, codes, scales, stream);
}

}  // extern "C"
