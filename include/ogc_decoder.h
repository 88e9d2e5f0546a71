/*
 * ogc_decoder.h -- C ABI of a decoder's attention block for AMD MI355X (gfx950): head norms with rotary positions, a key/value
 * cache held in 4 bits (written, read back), attention over that cache, and attention over packed prompts.
 *
 * They are meant to be used one after the other: the projection's queries and keys go through ogc_rope_run, the keys and the
 * values into the cache by ogc_kv4_write, and the queries meet the prompt's own keys (ogc_prompt_run) or, a few tokens of each
 * sequence at a time, the cache (ogc_kv4_attention_run).
 *
 * Rows and strides.  Tensors are DEVICE pointers to [rows][heads][head_dim] with element (row, head, channel) at
 *     base + row*stride[0] + head*stride[1] + channel      (strides in elements, channels contiguous)
 * so that the slices of one projection's output work as they are.  Strides are multiples of 16 bytes, bases 16-byte aligned.
 * The rows of several sequences are packed: sequence b has the rows cu[b] .. cu[b + 1] - 1 (cu: device int32 [batch + 1], ascending
 * from 0).  The number of rows and the longest sequence are given by the host, because launches are sized by them: a sequence's rows
 * beyond the longest that was announced are left out (a prompt's keys are not), and indices beyond the number of rows are cut to it.
 *
 * Types: OGC_F32 and OGC_BF16.  Sums, norms, softmax statistics and angles are held in 32 bits or more; bf16 results are rounded once,
 * to nearest even.  head_dim is 32, 64, 96 or 128, of all operators.
 *
 * Every call is asynchronous on `stream` (a hipStream_t, NULL = the default stream) and may be captured into a graph; the library
 * allocates nothing and keeps nothing between calls.  Errors are return codes (ogc_status of ogc_mlp.h), found before any
 * launch: OGC_ERR_INVALID_ARG (NULL, an unknown enum, a scalar out of range), OGC_ERR_SHAPE (sizes), OGC_ERR_UNSUPPORTED (dtype,
 * head_dim), OGC_ERR_ALIGNMENT (strides, pointers), OGC_ERR_DEVICE (a launch failed).  Calls without rows do nothing.
 */
#ifndef OGC_DECODER_H
#define OGC_DECODER_H

#include "ogc_mlp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- norms of queries and keys for each head, with the rotation of their positions in the same pass ----------------------------
 * For every row and head of q (and k alike, with k_weight):
 *     x = norm ? q * rsqrt(mean_c(q[c]^2) + eps) * q_weight[c] : q                fp32
 *     pairs (a, b) of the first rot_dim channels: (a cos - b sin, a sin + b cos)   angle = positions[row] * frequencies[pair]
 * OGC_ROPE_HALF pairs channels i and i + rot_dim/2, OGC_ROPE_INTERLEAVED 2i and 2i + 1.  The channels from rot_dim on are only
 * normed.  The angle is an fp64 product, reduced to a quarter turn in fp64: far positions keep their digits.  cosine and sine are
 * multiplied by `magnitude` (1, or what a stretched context asks for; stretching itself is the frequencies' business). */
typedef enum { OGC_ROPE_HALF = 0, OGC_ROPE_INTERLEAVED = 1 } ogc_rope_layout;

typedef struct ogc_rope_desc {
    int32_t dtype;
    int32_t tokens;             /* rows, >= 0 */
    int32_t q_heads, kv_heads;  /* > 0 */
    int32_t head_dim;
    int32_t rot_dim;            /* rotated channels: a multiple of 8, at most head_dim; 0: none */
    int32_t layout;             /* ogc_rope_layout */
    int32_t norm;               /* 1: norms, 0: none (eps and the weights are not looked at) */
    float eps;                  /* >= 0, finite */
    float magnitude;            /* finite */
    int64_t q_stride[2], k_stride[2], qo_stride[2], ko_stride[2]; /* row, head */
} ogc_rope_desc;

ogc_status ogc_rope_validate(const ogc_rope_desc* desc);
/* q_weight, k_weight: fp32 [head_dim], 16-byte aligned, unless norm is 0; positions: int32 [tokens]; frequencies: fp64 [rot_dim / 2], unless
 * rot_dim is 0.  q_out may be q and k_out may be k, with the same strides; other overlaps are not allowed. */
ogc_status ogc_rope_run(const ogc_rope_desc* desc, const void* q, const void* k, const float* q_weight, const float* k_weight,
                        const int32_t* positions, const double* frequencies, void* q_out, void* k_out, void* stream);

/* ---- the cache ---------------------------------------------------------------------------------------------------------------
 * uint8 [pages][kv_heads][page_size / 32][34 * head_dim]: a record for 32 tokens of a head with
 *     the keys' codes        [token][channel / 2]                                             16 head_dim bytes
 *     the values' codes      [channel / 32][token / 8][channel % 16][channel / 16 % 2][token % 8 / 2]   16 head_dim
 *     the keys' exponents    [channel / 32][token]                                            head_dim
 *     the values' exponents  [channel / 32][token]                                            head_dim
 * Even channels (values: even tokens) are in a byte's low half.  A code is E2M1 (sign, then 0, 1/2, 1, 3/2, 2, 3, 4, 6), and 32 channels
 * of a token share the scale 2^(byte - 127); byte 255 is no number.  The record's order is that of the matrix instruction's operands.
 * Token t of sequence b is at place t % page_size of the page page_table[b][t / page_size] (device int32 [batch][table_width]).  Entries
 * outside 0 .. pages - 1 stand for no page: what is written there is dropped, read back it is zero, and attention does not see it. */
typedef struct ogc_kv4_desc {
    int32_t kv_heads, head_dim; /* > 0 */
    int32_t page_size;          /* tokens, a multiple of 32 */
    int32_t pages;              /* > 0; of any total size */
    int32_t batch;              /* sequences, > 0 */
    int32_t table_width;        /* page table entries of a sequence, > 0; table_width * page_size at most 2^31 - 2^16 */
} ogc_kv4_desc;

/* Packed rows of keys and values, as they are written or read. */
typedef struct ogc_kv4_rows {
    int32_t dtype;
    int32_t rows, max_rows; /* of all sequences, of the longest; >= 0 */
    int64_t k_stride[2], v_stride[2];
} ogc_kv4_rows;

ogc_status ogc_kv4_validate(const ogc_kv4_desc* cache, const ogc_kv4_rows* rows);
ogc_status ogc_kv4_cache_bytes(const ogc_kv4_desc* cache, size_t* bytes);

/* Quantizes the rows cu[b] .. of k and v and stores them as the tokens start[b] .. of sequence b (start: device int32 [batch]).  The
 * scale is the smallest power of two at which the largest of 32 channels rounds to 6 or less, between 2^-127 and 2^125; codes
 * are rounded to nearest, ties to the even code, and end at 6 (which only magnitudes from 1.75 * 2^127 on exceed).  32 channels that hold an infinity or NaN are stored as no numbers.  All other
 * bytes of the cache stay as they are: an odd start keeps the token before it.  Pages of different sequences that are written must be
 * different ones.  cache: 16-byte aligned. */
ogc_status ogc_kv4_write(const ogc_kv4_desc* cache_desc, const ogc_kv4_rows* rows, const void* k, const void* v, const int32_t* cu,
                         const int32_t* start, const int32_t* page_table, void* cache, void* stream);
/* The values that tokens start[b] .. of sequence b have in the cache, into the rows cu[b] .. of k and v. */
ogc_status ogc_kv4_read(const ogc_kv4_desc* cache_desc, const ogc_kv4_rows* rows, const void* cache, const int32_t* cu,
                        const int32_t* start, const int32_t* page_table, void* k, void* v, void* stream);

/* ---- attention over the cache ------------------------------------------------------------------------------------------------
 * The last n = cu[b + 1] - cu[b] of the lens[b] tokens of sequence b ask: query i of them sees the tokens 0 .. lens[b] - n + i.
 *     o[i] = sum_j p[j] v[j] / sum_j p[j],   p[j] = exp(scale * q[i] . k[j] - reference)
 * Query heads h * q_heads / kv_heads .. share the key head h.  Products of bf16 values with fp32 sums (codes times a power of two
 * are bf16 values as they are); OGC_BF16 rounds the weights to bf16 for the second product and adds up the rounded ones, OGC_F32
 * splits queries and weights into three bf16 values, without loss but for channels of a query below 2^-64 of its largest one.  A query that
 * sees nothing gets zeros.  Values whose scale is 2^-127 count as zero here. */
typedef struct ogc_kv4_attention_desc {
    int32_t dtype;          /* of q and o */
    int32_t q_heads;        /* a multiple of kv_heads, at most 256 times it */
    int32_t rows, max_rows; /* queries of all sequences, of the one with most; >= 0 */
    int32_t max_keys;       /* tokens of the longest sequence, >= 0: longer ones are cut to it */
    float scale;            /* 2^-60 .. 2^60 */
    int64_t q_stride[2], o_stride[2];
} ogc_kv4_attention_desc;

ogc_status ogc_kv4_attention_validate(const ogc_kv4_desc* cache_desc, const ogc_kv4_attention_desc* desc);
/* Bytes that a call needs at `workspace` (0: none), for sequences shared by several workgroups.  They are enough for the same call with
 * fewer max_keys, too: a workspace for the longest that a cache will hold can be kept as it fills. */
ogc_status ogc_kv4_attention_workspace_bytes(const ogc_kv4_desc* cache_desc, const ogc_kv4_attention_desc* desc, size_t* bytes);
/* q, o: packed rows; o is written for all of them and must not overlap the inputs.  lens: device int32 [batch].  workspace: 16-byte
 * aligned, contents do not matter. */
ogc_status ogc_kv4_attention_run(const ogc_kv4_desc* cache_desc, const ogc_kv4_attention_desc* desc, const void* q, const int32_t* cu,
                                 const int32_t* lens, const int32_t* page_table, const void* cache, void* o, void* workspace,
                                 void* stream);

/* ---- attention over packed prompts -------------------------------------------------------------------------------------------
 * Sequence b has the queries cu_q[b] .. cu_q[b + 1] - 1 and the keys and values cu_k[b] .. cu_k[b + 1] - 1.  Causal: the queries are the
 * last ones of the sequence, query i of n sees the keys 0 .. m - n + i of m.  Query heads share key heads as above.  A query that
 * sees nothing (more queries than keys, or no keys) gets zeros; keys and values that a query does not see have no part in its result,
 * whatever they hold.  Arithmetic as ogc_mha_run of ogc_mha.h, stable softmax. */
typedef struct ogc_prompt_desc {
    int32_t dtype;
    int32_t batch;              /* > 0 */
    int32_t q_heads, kv_heads;  /* > 0; q_heads a multiple of kv_heads, at most 256 times it */
    int32_t head_dim;
    int32_t q_rows, k_rows;     /* of all sequences, >= 0 */
    int32_t max_q, max_k;       /* of the longest, >= 0; max_k orders the work and no more: keys beyond it are seen, and too large a one costs nothing */
    float scale;                /* 2^-60 .. 2^60 */
    int32_t causal;             /* 1, or 0: every query sees every key of its sequence */
    int64_t q_stride[2], k_stride[2], v_stride[2], o_stride[2];
} ogc_prompt_desc;

ogc_status ogc_prompt_validate(const ogc_prompt_desc* desc);
/* o is written for every query and must not overlap the inputs. */
ogc_status ogc_prompt_run(const ogc_prompt_desc* desc, const void* q, const void* k, const void* v, const int32_t* cu_q,
                          const int32_t* cu_k, void* o, void* stream);
/* Name of the kernel that ogc_prompt_run launches for this description, as a kernel trace prints it (static storage), or NULL. */
const char* ogc_prompt_kernel_name(const ogc_prompt_desc* desc);

#ifdef __cplusplus
}
#endif
#endif
