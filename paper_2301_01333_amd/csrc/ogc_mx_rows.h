// Eight channels of a row, as they are in memory and in fp32, and their way into a microscaled format: what the norm and the operators on rows
// share.
#ifndef OGC_MX_ROWS_H
#define OGC_MX_ROWS_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ogc_mlp.h"
#include "ogc_mx.h"
#include "ogc_mx_layout.h"

#define MX_DEV static __device__ __forceinline__

typedef float mx_v2f __attribute__((ext_vector_type(2)));
typedef float mx_v4f __attribute__((ext_vector_type(4)));
typedef uint32_t mx_v2u __attribute__((ext_vector_type(2)));
typedef uint32_t mx_v4u __attribute__((ext_vector_type(4)));
typedef uint32_t mx_v4u_anywhere __attribute__((ext_vector_type(4), aligned(2)));  // (loaded by the same instruction as an aligned one)
typedef __bf16 mx_v2bf __attribute__((ext_vector_type(2)));
typedef short mx_v2s __attribute__((ext_vector_type(2)));

template <int DT> struct MxEight {
    static constexpr int E = DT == OGC_F32 ? 4 : 2;
    mx_v4u raw[DT == OGC_F32 ? 2 : 1];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < (DT == OGC_F32 ? 2 : 1); ++i) raw[i] = (mx_v4u){0, 0, 0, 0};
    }
    // the first `there` of the eight channels at p, zeros for the others; nothing else is touched
    __device__ __forceinline__ void load(const uint8_t* p, int there) {
        if (there >= 8) {
            raw[0] = *(const mx_v4u_anywhere*)p;
            if constexpr (DT == OGC_F32) raw[1] = *(const mx_v4u_anywhere*)(p + 16);
        } else {
            clear();
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < there) {
                    if constexpr (DT == OGC_F32) raw[i / 4][i % 4] = *(const uint32_t*)(p + 4 * i);
                    else raw[0][i / 2] |= (uint32_t) * (const uint16_t*)(p + 2 * i) << (i % 2 * 16);
                }
        }
    }
    __device__ __forceinline__ void store(uint8_t* p, int there) const {
        if (there >= 8) {
            *(mx_v4u*)p = raw[0];
            if constexpr (DT == OGC_F32) *(mx_v4u*)(p + 16) = raw[1];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < there) {
                    if constexpr (DT == OGC_F32) *(uint32_t*)(p + 4 * i) = raw[i / 4][i % 4];
                    else *(uint16_t*)(p + 2 * i) = (uint16_t)(raw[0][i / 2] >> (i % 2 * 16));
                }
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (DT == OGC_F32) return __builtin_bit_cast(float, (uint32_t)raw[i / 4][i % 4]);
        else return __builtin_bit_cast(float, i & 1 ? (uint32_t)raw[0][i / 2] & 0xffff0000u : (uint32_t)raw[0][i / 2] << 16);
    }
    __device__ __forceinline__ void next() {  // channel 1 in the place of channel 0, and so on
        if constexpr (DT == OGC_F32) {
            const uint32_t first = raw[0][0];
            raw[0] = (mx_v4u){raw[0][1], raw[0][2], raw[0][3], raw[1][0]};
            raw[1] = (mx_v4u){raw[1][1], raw[1][2], raw[1][3], first};
        } else {
            const mx_v4u t = raw[0];
            raw[0] = (mx_v4u){t[0] >> 16 | t[1] << 16, t[1] >> 16 | t[2] << 16, t[2] >> 16 | t[3] << 16, t[3] >> 16 | t[0] << 16};
        }
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {  // bf16: rounded to nearest even
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            if constexpr (DT == OGC_F32) {
                raw[i / 4][i % 4] = __builtin_bit_cast(uint32_t, x[i]);
                raw[i / 4][i % 4 + 1] = __builtin_bit_cast(uint32_t, x[i + 1]);
            } else {
                const mx_v2bf t = {(__bf16)x[i], (__bf16)x[i + 1]};
                raw[0][i / 2] = __builtin_bit_cast(uint32_t, t);
            }
        }
    }
};

template <int CTRL> MX_DEV uint32_t mx_quad(uint32_t x) { return __builtin_amdgcn_mov_dpp(x, CTRL, 0xf, 0xf, true); }

// Codes and exponent of eight channels, in two words (FORMAT OGC_MX4: the first).  Four neighbouring lanes, from a multiple of four on, hold a group; all 64 lanes take part.
template <int FORMAT> MX_DEV mx_v2u mx_quantized(const float (&x)[8], uint32_t& exponent) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);
    top = max(top, mx_quad<0xB1>(top));  // lane ^ 1
    top = max(top, mx_quad<0x4E>(top));  // lane ^ 2
    // E2M1: up to 7 (exclusive) times the scale rounds to 6, so that mantissas from 1.75 on take the next power; E4M3: up to 464 (inclusive)
    // to 448, mantissas beyond 1.8125
    const int e = FORMAT == OGC_MX4 ? (int)((top + 0x200000u) >> 23) - 2 : (int)((top + 0x17ffffu) >> 23) - 8;
    const bool number = top < 0x7f800000u;
    exponent = number ? min(max(e, 0), FORMAT == OGC_MX4 ? 252 : 246) : 255;
    const float scale = __builtin_bit_cast(float, exponent << 23);  // (the instruction takes the exponent's bits: 0 is 2^-127)
    // (only groups that would need a larger scale than there is have more than this)
    const float most = FORMAT == OGC_MX4 ? 0x1.8p127f : 0x1.cp127f;
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = __builtin_amdgcn_fmed3f(x[i], -most, most);
    mx_v2u code = {0, 0};
    if constexpr (FORMAT == OGC_MX4) {
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, z[0], z[1], scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, z[2], z[3], scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, z[4], z[5], scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, z[6], z[7], scale, 3);
        code[0] = number ? c : 0;
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            mx_v2s c = {0, 0};
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, z[4 * h], z[4 * h + 1], scale, false);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, z[4 * h + 2], z[4 * h + 3], scale, true);
            code[h] = number ? __builtin_bit_cast(uint32_t, c) : 0;
        }
    }
    return code;
}

#endif
