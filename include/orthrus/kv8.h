/*
 * orthrus/kv8.h -- an 8-bit paged KV cache and the operators on it: head norms, rotation and
 * append, read-back, and causal attention of ragged rows (single tokens, few tokens, prompt
 * chunks).  Conventions (ownership, streams, status codes) are those of orthrus.h.
 *
 * What the cache holds.  A page is 16 consecutive positions of one sequence.  Keys and values are
 * stored as 8-bit floats (e4m3: 4 exponent, 3 mantissa bits, largest value 448, no infinities)
 * with one fp32 scale for each page and KV head, keys and values apart; the value of a code is
 * code * scale.  Scales are powers of two, so a code's value is exact in bfloat16.
 *   - Appending rounds to nearest, ties to even, under the least scale 2^e (e >= -100) with
 *     max |x| <= 448 * 2^e over the finite elements of the page's tokens so far.
 *   - While a page fills, its scale never shrinks.  Where a token needs a larger one, the codes
 *     that the page already holds are rounded again under it.
 *   - A position at the start of a page forgets what the page held before.  Appending before positions that the page
 *     holds gives those up: their codes stay, but not their scale.
 *   - Elements that are infinite or not a number, or that would round to 2^128 (magnitudes from 1.9375 * 2^127 on, which
 *     count as infinite), are stored as not a number.
 */
#ifndef ORTHRUS_KV8_H
#define ORTHRUS_KV8_H

#include "../orthrus.h"

#ifdef __cplusplus
extern "C" {
#endif

/* device error bit: a call used a workspace that holds another plan (see orthrus_rows_plan) */
#define ORTHRUS_DEVERR_STALE 4

/* The cache (device).  Pools: k [n_layers][n_pages][n_kv_heads][16][head_dim] and
 * v [n_layers][n_pages][n_kv_heads][4][16][head_dim / 16][4] one-byte codes, 16-byte aligned: the
 * values of one page and head lie by [slot / 4][dim % 16][dim / 16][slot % 4], so that the four
 * slots of a dim and the eight dims a lane multiplies are one contiguous run.  Scales:
 * [n_layers][n_pages][n_kv_heads] fp32.  block_table: int32 [n_seq][max_blocks]; position p of
 * sequence s lives in page block_table[s][p / 16], slot p % 16. */
typedef struct orthrus_kv8 {
    void *k_cache, *v_cache;
    float *k_scale, *v_scale;
    const int32_t *block_table;
    int32_t n_layers, n_pages, n_seq, max_blocks;
} orthrus_kv8;

/* The heads of a layer.  Supported: head_dim 64 or 128, any group n_q_heads / n_kv_heads of 1 to
 * 16, page_size 16.  dtype (ORTHRUS_F32 or ORTHRUS_BF16): element type of q, of the rotated q that
 * append writes and of the attention output.
 * Rotation: the leading rot_dims dims of q and k turn (a multiple of 16 up to head_dim; 0: none),
 * in pairs (i, i + rot_dims / 2), or (2 i, 2 i + 1) if interleaved.  Pair i of position p turns by
 * the angle p * f_i, f_i = rope_freq[i] if rope_freq (HOST, rot_dims / 2 doubles, copied) is given,
 * else rope_base^(-2 i / rot_dims); angles are evaluated in double.  Cosine and sine are multiplied
 * by rope_magnitude (1 where positions are not scaled).
 * norm_eps: added to the mean square of a head where orthrus_kv8_append is given a gain. */
typedef struct orthrus_head_shape {
    int32_t n_q_heads, n_kv_heads, head_dim, page_size, dtype;
    int32_t rot_dims, interleaved;
    float rope_base, rope_magnitude, norm_eps;
    const double *rope_freq;
} orthrus_head_shape;

/* One segment: the tokens at positions [offset, offset + len) of sequence `seq`, as consecutive
 * rows of the call's tensors.  A decode row is a segment of one token. */
typedef struct orthrus_segment {
    int32_t seq, offset, len;
} orthrus_segment;

/* Host handle: the head shape and the plan of the rows that the calls below work on. */
typedef struct orthrus_rows orthrus_rows;

/* Validates and copies `shape` (EINVAL / EUNSUPPORTED).  No device work. */
int orthrus_rows_create(const orthrus_head_shape *shape, orthrus_rows **out);
void orthrus_rows_destroy(orthrus_rows *r);

/* Device workspace bytes for plans of at most max_rows rows in at most max_segments segments that
 * see at most max_keys positions each (offset + len).  0 for invalid arguments. */
size_t orthrus_rows_workspace_bytes(const orthrus_rows *r, int32_t max_rows, int32_t max_segments, int32_t max_keys);

/* Plans the rows of the following calls: segment i's rows follow segment i - 1's.  Validates before
 * anything is enqueued: EDESC (seq outside [0, n_seq), offset < 0, len < 1), EDUPSEQ (a sequence in
 * two segments), ECAPACITY (past the block table, more than 2^23 rows times KV heads, or workspace too small),
 * EUNSUPPORTED (stream under capture).  Sequences may share pages that are only read; the pages that one segment
 * appends to are no other segment's.  Uploads the plan into `workspace` (256-byte aligned, cleared once by
 * orthrus_workspace_init) on `stream`; n = 0 is a plan without rows.
 * The plan holds until the next one of this handle, for any layer of any cache that has its
 * sequences.  The handle belongs to the device that is current at its first plan (EINVAL on another).
 * The calls below read plan and partial results from the workspace: one call in flight per
 * workspace.  They may be captured into a graph, which replays the plan it was captured with; once
 * the workspace holds another plan, a replay does nothing but set ORTHRUS_DEVERR_STALE (read and cleared by
 * orthrus_device_error(workspace, ...), like ORTHRUS_DEVERR_PAGE).  Not thread-safe per handle. */
int orthrus_rows_plan(orthrus_rows *r, const orthrus_kv8 *kv, const orthrus_segment *segments, int32_t n, void *workspace,
                      size_t ws_bytes, void *stream);

/* The attention work of a plan without touching the GPU (for inspection and tests): validates like
 * orthrus_rows_plan and writes up to `cap` items of 8 int32:
 *   {sequence, first row, rows, position of the first row, KV head, key begin, key end, partial slot or -1};
 * counts: {items of few rows (rows * group <= 16), items of more rows, merges, partial slots of 16 rows}. */
int orthrus_rows_items(const orthrus_rows *r, const orthrus_kv8 *kv, const orthrus_segment *segments, int32_t n,
                       int32_t counts[4], int32_t *items, int32_t cap);

/* Norm, rotation and append of the planned rows in layer `layer`.  qkv: device [rows][row_stride] of
 * qkv_dtype, each row the query heads, then the key heads, then the value heads.  q_gain, k_gain:
 * fp32 device [head_dim] or NULL: a head x becomes x * gain / sqrt(mean(x^2) + norm_eps) before it
 * turns.  q_out: device [rows][q_stride] of the shape's dtype: the rotated query heads.  Keys (rotated) and
 * values are appended at the rows' positions.  Strides in elements, multiples of 8, at least
 * (n_q + 2 n_kv) head_dim and n_q head_dim; bases 16-byte aligned (EINVAL).  qkv_dtype ORTHRUS_BF16 needs a
 * shape of that dtype (EUNSUPPORTED).  q_out may be the rows' own query columns (base, stride and type of qkv); else
 * it shares no element with them.  A page id outside [0, n_pages) sets ORTHRUS_DEVERR_PAGE and its
 * tokens are not stored. */
int orthrus_kv8_append(const orthrus_rows *r, const orthrus_kv8 *kv, int32_t layer, const void *qkv, int32_t qkv_dtype,
                       int64_t row_stride, const float *q_gain, const float *k_gain, void *q_out, int64_t q_stride,
                       void *stream);

/* The values that the cache holds at the planned rows' positions, exact in bfloat16: k_out, v_out device
 * [rows][n_kv head_dim], 16-byte aligned.  Rows of bad pages are zero (ORTHRUS_DEVERR_PAGE). */
int orthrus_kv8_read(const orthrus_rows *r, const orthrus_kv8 *kv, int32_t layer, void *k_out, void *v_out, void *stream);

/* Causal attention of the planned rows over the cache in layer `layer`: the row at position p of its
 * sequence sees positions 0 .. p (its own key and value appended before); query head h reads KV
 * head h / (n_q / n_kv).  out = softmax(scale * q k^T) v; scale 0 means 1 / sqrt(head_dim) (EINVAL if
 * negative, or not finite once multiplied by log2(e)).  q, out: device [rows][stride] of the shape's dtype, n_q head_dim values a
 * row; strides multiples of 8 elements, bases 16-byte aligned (EINVAL); out may be q itself (base and stride), else the
 * two share no element.  Scores, softmax and sums in
 * fp32; bfloat16 rows round the softmax weights to bfloat16 before the product with the values and divide by the sum
 * of the rounded ones, fp32 rows keep them whole.  Keys of a page outside [0, n_pages) are skipped (ORTHRUS_DEVERR_PAGE); a row
 * left without keys is zero.  A row that sees only scores of minus infinity is not a number, as its softmax. */
int orthrus_kv8_attend(const orthrus_rows *r, const orthrus_kv8 *kv, int32_t layer, const void *q, int64_t q_stride,
                       float scale, void *out, int64_t out_stride, void *stream);

/* One mixed step (orthrus_step) through 8-bit caches: the same batch, models, pooling, outputs and status codes, with
 * keys and values appended to and read from emb_kv and gen_kv by the operators above (rotation as the model's: half
 * pairs of whole heads).  The models' heads are within the limits of orthrus_rows_create and the rows within those of
 * orthrus_rows_plan; nothing is enqueued where they are not.  A cache has the models' KV heads and head dimension, at
 * least as many layers (EINVAL), and its pools are given also where a model has no layers.  gen_kv may be emb_kv, or
 * equal to it in every field: then all items share one sequence namespace.  Pools and scales, of two caches
 * or of one, do not overlap (EINVAL).  workspace: 256-byte aligned, at least orthrus_step_kv8_bytes() for this batch's
 * sizes (arguments as those of orthrus_workspace_bytes; a chunk's end counts as a context for max_ctx), cleared once by
 * orthrus_workspace_init; its error word (orthrus_device_error) also gets the operators' bits.  Host sides of calls that
 * share `emb` run one after the other; one step in flight per workspace.  Not for capture into a HIP graph (EUNSUPPORTED). */
size_t orthrus_step_kv8_bytes(const orthrus_model *emb, const orthrus_model *gen, int32_t max_tokens, int32_t max_chunks,
                              int32_t max_decode, int32_t max_ctx);
int orthrus_step_kv8(const orthrus_model *emb, const orthrus_model *gen, const orthrus_batch *batch, const orthrus_kv8 *emb_kv,
                     const orthrus_kv8 *gen_kv, float *acc_sum, float *acc_w, float *out_logits, float *out_emb, void *workspace,
                     size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ORTHRUS_KV8_H */
