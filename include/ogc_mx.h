/*
 * ogc_mx.h -- C ABI of a decoder's projections in microscaled formats for AMD MI355X (gfx950): the residual's addition with the
 * root-mean-square norm, rows written in a microscaled format and read back, and the product of such rows with 4-bit weights.
 *
 * They are meant to be used one after the other: ogc_norm_run leaves a layer's rows in 8 or 4 bits with scales, ogc_mx_product_run takes them
 * to the next projection, ogc_mx_write does the same for what attention or a gate leaves, and lays out weights.  The residual
 * meets the projection's result in the next norm.
 *
 * A microscaled matrix.  32 channels of a row, a group, share the scale 2^(byte - 127); byte 255 is no number.  Rows are rounded up to 32 and
 * channels to 256, and all of it is in the order of the matrix instruction's operands:
 *     OGC_MX4  codes E2M1 (sign, then 0, 1/2, 1, 3/2, 2, 3, 4, 6), two a byte, even channels in the low half
 *              [rows / 32][channels / 32][32 rows][16 bytes]
 *     OGC_MX8  codes E4M3 (largest 448, as OGC_F8 of ogc_mlp.h)
 *              [rows / 32][channels / 16][32 rows][16 bytes]
 *     scales   [rows / 32][channels / 256][2][32 rows][4 bytes]: group 2 i + j of eight is at [j][row][i]
 * What is written here has zero codes in the channels that were rounded up; their scales are no 255.  The rows that were
 * rounded up are left as they were, and no result depends on them.  ogc_mx_bytes gives the sizes; codes and scales are 16-byte aligned.
 *
 * Other tensors are DEVICE pointers to rows of contiguous channels, a stride apart (in elements; a multiple of 16 bytes; bases 16-byte aligned).
 * Rows that are read may overlap (a stride of 0 is the same row again), rows that are written must not.
 * Types: OGC_F32 and OGC_BF16.  Sums are held in 32 bits (the norm's in 64); results are rounded once, to nearest even.
 *
 * Every call is asynchronous on `stream` (a hipStream_t, NULL = the default stream) and may be captured into a graph; the library
 * allocates nothing and keeps nothing between calls.  Errors are return codes (ogc_status of ogc_mlp.h), found before any
 * launch: OGC_ERR_INVALID_ARG (NULL, an unknown enum, a scalar out of range), OGC_ERR_SHAPE (sizes), OGC_ERR_UNSUPPORTED (types),
 * OGC_ERR_ALIGNMENT (strides, pointers), OGC_ERR_DEVICE (a launch failed).  Calls without rows do nothing.
 */
#ifndef OGC_MX_H
#define OGC_MX_H

#include "ogc_mlp.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { OGC_MX4 = 0, OGC_MX8 = 1 } ogc_mx_format;

/* Bytes of a matrix's codes and scales.  rows >= 0, channels > 0. */
ogc_status ogc_mx_bytes(int32_t format, int32_t rows, int32_t channels, size_t* codes, size_t* scales);

/* ---- the residual's addition with the root-mean-square norm ----------------------------------------------------------------------
 * For every row:   s = x + residual, rounded to the type (no residual: s = x)
 *                  y = s * rsqrt(mean_c(s[c]^2) + eps) * weight[c]
 * s is kept as the next residual.  Squares and their sum are held in 64 bits, so that rows of all numbers have their norm; the factor is rounded to fp32.  OGC_NORM_SAME: y in the type of x; OGC_NORM_MX4, OGC_NORM_MX8: y as a microscaled matrix, quantized from its
 * fp32 values as by ogc_mx_write. */
typedef enum { OGC_NORM_SAME = 0, OGC_NORM_MX4 = 1, OGC_NORM_MX8 = 2 } ogc_norm_out;

typedef struct ogc_norm_desc {
    int32_t dtype;
    int32_t rows, channels;     /* rows >= 0, below 2^22; channels > 0, at most 2^20 */
    int32_t out;                /* ogc_norm_out */
    float eps;                  /* >= 0, finite */
    int64_t x_stride, residual_stride, sum_stride, y_stride; /* the residual's and the sum's: 0 without one; y's: OGC_NORM_SAME */
} ogc_norm_desc;

ogc_status ogc_norm_validate(const ogc_norm_desc* desc);
/* residual: or NULL, then sum is not written and may be NULL.  weight: fp32 [channels], 16-byte aligned.  y: rows, or the matrix's codes with
 * `scales`.  sum may be x or residual, or y (OGC_NORM_SAME) may be x, with the same strides; other overlaps are not allowed. */
ogc_status ogc_norm_run(const ogc_norm_desc* desc, const void* x, const void* residual, const float* weight, void* sum, void* y,
                        void* scales, void* stream);

/* ---- rows in microscaled formats -------------------------------------------------------------------------------------------------
 * The scale of a group is the smallest power of two, from 2^-127, at which the largest of its 32 values rounds to 6 (OGC_MX8: 448) or less; codes
 * are rounded to nearest, ties to the even code.  The largest scales are 2^125 (2^119): magnitudes that would need more end at
 * 6 (448) times that.  A group that holds an infinity or NaN is stored as no numbers: byte 255, codes zero.
 * OGC_GATE_SILU: rows of 2 * channels, and a * b / (1 + exp(-a)) is written, a = channel c, b = channel channels + c, in fp32. */
typedef enum { OGC_GATE_NONE = 0, OGC_GATE_SILU = 1 } ogc_gate;

typedef struct ogc_mx_rows {
    int32_t dtype;
    int32_t format;             /* ogc_mx_format */
    int32_t rows, channels;     /* rows >= 0; channels > 0, at most 2^20; (rows / 32) * (channels / 256), rounded up, below 2^24 */
    int32_t gate;               /* ogc_gate; ogc_mx_read: OGC_GATE_NONE */
    int64_t stride;             /* of the rows of x or y */
} ogc_mx_rows;

ogc_status ogc_mx_validate(const ogc_mx_rows* rows);
ogc_status ogc_mx_write(const ogc_mx_rows* rows, const void* x, void* codes, void* scales, void* stream);
/* The values that the rows have in the matrix, rounded to the type (OGC_BF16 holds all of them that are not below its smallest one). */
ogc_status ogc_mx_read(const ogc_mx_rows* rows, const void* codes, const void* scales, void* y, void* stream);

/* ---- product ---------------------------------------------------------------------------------------------------------------------
 * y[i][j] = sum_c x[i][c] w[j][c] + bias[j],  x [m][k] and w [n][k] microscaled matrices.  Products are exact; those of eight neighbouring channels are added without
 * loss, these sums in fp32, 8-bit rows as two sums each (codes below 2 and the others).  Only bf16 results of OGC_MX8 rows may have less, where a call has many rows (ogc_mx_product_kernel_name: not
 * ogc_mx_few_kernel<.., 1>): of eight products what is below 2^-14 of the largest one's power of two is dropped (measured: 4e-6 of a result of random rows). */
typedef struct ogc_mx_product_desc {
    int32_t dtype;              /* of y */
    int32_t x_format, w_format; /* OGC_MX4 or OGC_MX8; OGC_MX4 */
    int32_t m, n, k;            /* m >= 0; n, k > 0; at most 2^21, 2^26, 2^20, and (m / 256) * (n / 256), rounded up, 2^23 - 8 */
    int32_t has_bias;           /* 0 or 1 */
    int64_t y_stride;
} ogc_mx_product_desc;

ogc_status ogc_mx_product_validate(const ogc_mx_product_desc* desc);
/* Bytes that a call needs at `workspace`: 0, for every description.  (The product has the form of the calls that do need one.) */
ogc_status ogc_mx_product_workspace_bytes(const ogc_mx_product_desc* desc, size_t* bytes);
/* bias: fp32 [n], 4-byte aligned, unless has_bias is 0.  y must not overlap the inputs.  workspace: not looked at, and may be NULL. */
ogc_status ogc_mx_product_run(const ogc_mx_product_desc* desc, const void* x, const void* x_scales, const void* w, const void* w_scales,
                              const float* bias, void* y, void* workspace, void* stream);
/* Name of the kernel that ogc_mx_product_run launches for this description, as a kernel trace prints it (static storage), or NULL. */
const char* ogc_mx_product_kernel_name(const ogc_mx_product_desc* desc);

#ifdef __cplusplus
}
#endif
#endif
