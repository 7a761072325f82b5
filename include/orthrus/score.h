/*
 * orthrus/score.h -- scores of tokens under the logits that orthrus_step() writes, beside the greedy
 * sampler of orthrus.h; conventions are those of orthrus.h.
 */
#ifndef ORTHRUS_SCORE_H
#define ORTHRUS_SCORE_H

#include "../orthrus.h"

#ifdef __cplusplus
extern "C" {
#endif

/* most entries n_top of orthrus_logprobs */
#define ORTHRUS_MAX_TOP 64

/* Device workspace bytes of orthrus_logprobs for these sizes (0 for invalid ones). */
size_t orthrus_logprobs_bytes(int32_t rows, int32_t vocab, int32_t n_top);

/* Scores of one token a row and the row's largest entries, enqueued on `stream`.  For row r with
 * logits x (fp32 device, row_stride >= vocab elements apart) and Z = sum_v exp(x_v):
 *   logprob[r]  = x_t - log Z of t = tokens[r] (int32 device);
 *   entropy[r]  = log Z - sum_v exp(x_v) x_v / Z, an entry of -inf counting 0;
 *   rank[r]     = number of entries that come before t: larger ones and equal ones of a lower index
 *                 (the order of orthrus_sample_greedy: a NaN is larger than every number);
 *   top_ids[r][j], top_logprobs[r][j]: entry j in that order and its log probability, j < n_top.
 * tokens may be NULL if logprob and rank are; a token outside [0, vocab) has logprob NaN and rank
 * -1.  Any output may be NULL and is then not written (top_ids and top_logprobs only with n_top = 0 both).  A row
 * with a NaN, with +inf, or of nothing but -inf has no distribution: its logprob, entropy and
 * top_logprobs are NaN, its rank and top_ids as ordered.  Sums are taken in fp32 in a fixed order.
 * workspace: device, orthrus_logprobs_bytes(), 16-byte aligned, one call in flight; may be NULL if that is 0.
 * EINVAL: negative sizes, vocab < 1, n_top outside [0, min(vocab, ORTHRUS_MAX_TOP)], row_stride < vocab, a null
 * pointer that is needed; ECAPACITY: ws_bytes too small, 2^22 or more rows (or rows times slices of 32 k entries)
 * or more than 2^30 entries a row.  rows = 0 is a no-op. */
int orthrus_logprobs(const float *logits, int64_t row_stride, int32_t rows, int32_t vocab, const int32_t *tokens,
                     int32_t n_top, float *logprob, float *entropy, int32_t *rank, int32_t *top_ids, float *top_logprobs,
                     void *workspace, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ORTHRUS_SCORE_H */
