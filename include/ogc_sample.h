/*
 * ogc_sample.h -- C ABI of the choice of a token from its logits for AMD MI355X (gfx950): temperature, top-k, top-p and min-p, from given
 * random numbers.
 *
 * For every row of logits (OGC_F32 or OGC_BF16, DEVICE pointer, rows a stride of elements apart):
 *     w[i] = exp((logit[i] - largest) / temperature)            tokens of -infinity and NaN have none
 *     in the order of falling logits (equal ones: the lowest index first),
 *         top_k: the first top_k tokens are kept;
 *         top_p: of these, the fewest first ones whose weights add up to top_p times the weight of all of these, or more;
 *         min_p: of these, the ones with w >= min_p (1 at most: the first token is always kept);
 *     the token is the first kept one, by index, at which the running sum of the kept weights exceeds uniform * their sum
 *     its log-probability is log(w / their sum).
 * temperature 0, below or NaN: the largest logit, the lowest index of equal
 * ones, with log-probability 0.  top_k <= 0, top_p >= 1 or NaN, min_p <= 0 or
 * NaN: no such limit.  A uniform below 0 or NaN counts as 0, one from 1 on takes the last kept token.  Logits of +infinity share the choice
 * among them.  A row without any token: -1, with log-probability -infinity.
 * Weights are computed in 64 bits and rounded to multiples of 2^-42 of the largest one of the row, or of a part of it (a token of less than 2^-43 of that has none).
 * They are added up as whole numbers, or in a fixed order, so that a call gives the same tokens every time; a decision that is closer than
 * vocab * 2^-42 of the sum it is compared with may fall either way.
 *
 * Calls are asynchronous on `stream` (a hipStream_t, NULL = the default stream) and may be captured into a graph; the library allocates nothing and keeps
 * nothing between calls.  Errors are return codes as in ogc_mx.h, found before any launch.  Calls without rows do nothing.
 */
#ifndef OGC_SAMPLE_H
#define OGC_SAMPLE_H

#include "ogc_mlp.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ogc_sample_desc {
    int32_t dtype;
    int32_t rows, vocab;        /* rows >= 0, at most 65535; vocab > 0, at most 2^20 */
    int64_t stride;             /* elements; any from vocab on */
} ogc_sample_desc;

ogc_status ogc_sample_validate(const ogc_sample_desc* desc);
/* Bytes that a call needs at `workspace` (0: none): half a byte for each logit, and 8 KiB for every 2048 to 8192 of a row. */
ogc_status ogc_sample_workspace_bytes(const ogc_sample_desc* desc, size_t* bytes);
/* logits: of any alignment of their type, and of any stride: rows are read 16 bytes at a time either way.  temperature, top_p, min_p, uniform: fp32 [rows], top_k: int32 [rows]; each but `uniform` may
 * be NULL (temperature 1, no limit).  tokens: int32 [rows]; log_probabilities: fp32 [rows], or NULL.  workspace: 16-byte aligned, contents do
 * not matter; calls that may run at the same time need different ones. */
ogc_status ogc_sample_run(const ogc_sample_desc* desc, const void* logits, const float* temperature, const int32_t* top_k,
                          const float* top_p, const float* min_p, const float* uniform, int32_t* tokens, float* log_probabilities,
                          void* workspace, void* stream);

#ifdef __cplusplus
}
#endif
#endif
