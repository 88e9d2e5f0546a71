// Where the codes and scales of a microscaled matrix are (include/ogc_mx.h), as plain arithmetic: used by the kernels, and by a test on the
// host that compares it with the documented order.
#ifndef OGC_MX_LAYOUT_H
#define OGC_MX_LAYOUT_H

#include <stdint.h>

#ifdef __HIP__
#define MX_FN static __host__ __device__ __forceinline__
#else
#define MX_FN static inline
#endif

constexpr int MX_ROWS = 32, MX_GROUP = 32, MX_BLOCK = 256;  // rows and channels that a matrix is rounded up to; channels of a scale

MX_FN int64_t mx_padded_rows(int rows) { return ((int64_t)rows + MX_ROWS - 1) / MX_ROWS * MX_ROWS; }
MX_FN int mx_padded_channels(int channels) { return (channels + MX_BLOCK - 1) / MX_BLOCK * MX_BLOCK; }
// bytes of the codes of 32 rows; format 0: two codes a byte, 1: one.  Of their scales: `padded` as well.
MX_FN int64_t mx_codes_of_32(int format, int padded) { return (int64_t)padded * (format ? 32 : 16); }
// byte of the codes where a row's channels channel .. begin (a multiple of what 16 bytes hold, or inside of them a whole byte)
MX_FN int64_t mx_code_at(int format, int padded, int row, int channel) {
    const int byte = format ? channel : channel / 2;
    return row / MX_ROWS * mx_codes_of_32(format, padded) + byte / 16 * 512 + row % MX_ROWS * 16 + byte % 16;
}
// the four scales of the groups j, j + 2, j + 4, j + 6 of a block of 256 channels
MX_FN int64_t mx_scales_at(int padded, int row, int block, int j) {
    return row / MX_ROWS * (int64_t)padded + block * MX_BLOCK + j * 128 + row % MX_ROWS * 4;
}

#endif
