/*
 * orthrus/linear.h -- the products and norms of a layer as operators: RMS norm with the residual's
 * addition, matrix products with bias, activation and residual in their epilogue, the same for
 * ragged groups of rows that go through weights of their own, and the 8-bit blocks that these read
 * and write.  Conventions (ownership, streams, status codes) are those of orthrus.h.
 *
 * 8-bit blocks (ORTHRUS_MX8).  32 consecutive elements of a row (the last ones of a row may be
 * fewer) share a power-of-two scale, held as its biased exponent in one byte: 2^(byte - 127), 255 is
 * not a number.  An element is an e4m3 code (4 exponent, 3 mantissa bits, largest value 448, no
 * infinities) times its block's scale: exact in fp32 under bytes up to 246, in bfloat16 under bytes 3 to 246 (rounding to blocks
 * writes bytes 27 to 247, and no value past fp32's range).
 *   - Rounding to blocks takes the least scale 2^e (e >= -100) with max |x| <= 448 * 2^e over the
 *     block's finite elements, and the nearest code, ties to even.
 *   - Elements that are infinite or not a number, or that would round to 2^128, become the code of
 *     not a number.
 */
#ifndef ORTHRUS_LINEAR_H
#define ORTHRUS_LINEAR_H

#include "../orthrus.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element type of the operators below: 8-bit blocks */
#define ORTHRUS_MX8 2
#define ORTHRUS_MX8_BLOCK 32

/* activations, of fp32 values in fp32.  Errors relative to the result, |v| up to 80: silu 2^-21 + |v| 2^-23, gelu 2^-18 + v^2 2^-23 (v
 * above -13), its tanh form 2^-21 + |v + 0.044715 v^3| 2^-20; results below 2^-119 may be zero. */
#define ORTHRUS_ACT_NONE 0
#define ORTHRUS_ACT_RELU 1      /* max(v, 0)                                          */
#define ORTHRUS_ACT_SILU 2      /* v / (1 + exp(-v))                                  */
#define ORTHRUS_ACT_GELU 3      /* v / 2 * (1 + erf(v / sqrt(2)))                     */
#define ORTHRUS_ACT_GELU_TANH 4 /* v / 2 * (1 + tanh(sqrt(2 / pi) (v + 0.044715 v^3))) */

/* Rows of elements on the device.  ORTHRUS_F32, ORTHRUS_BF16: data, `stride` elements between rows; scale is
 * not read.  ORTHRUS_MX8: data holds codes, `stride` bytes between rows, and scale one byte a block,
 * `scale_stride` bytes between rows.  What is read or written is stated at each call; rows do not overlap. */
typedef struct orthrus_matrix {
    void *data, *scale;
    int64_t stride, scale_stride;
    int32_t dtype;
} orthrus_matrix;

/* y = x in y's type, element by element: F32 or BF16 to MX8, or MX8 to F32 or BF16 (others
 * EUNSUPPORTED).  x and y share no memory (EINVAL).  Any strides >= width (scales: >= ceil(width / 32)) and any
 * alignment to an element. */
int orthrus_convert(const orthrus_matrix *x, const orthrus_matrix *y, int32_t rows, int32_t width, void *stream);

/* RMS norm of each row, after the addition of a residual: s = x + add (fp32; add NULL: s = x),
 * total = s rounded to its type (total NULL: not written), y = s * gain / sqrt(mean(s^2) + eps) in y's type
 * (gain fp32 device [width]; NULL: ones).  x, add, total: F32 or BF16; y: F32, BF16 or MX8.  total
 * or y may be x or add itself (data, stride and dtype, not MX8); else what is written shares no byte with anything (EINVAL).
 * The mean is taken in 64 bits of s as fp32 holds it: y is off by at most 2^-22 of itself, and half a step of its type (squares whose sum
 * passes fp32's range make a row zero; 8-bit codes with three bits of mantissa are rounded once, from s before its rounding).  Any
 * strides >= width and any alignment to an element.
 * EINVAL: a null pointer, width < 1, eps negative or not a number; ECAPACITY: width > 2^30. */
int orthrus_norm(const orthrus_matrix *x, const orthrus_matrix *add, const orthrus_matrix *total, const float *gain, float eps,
                 const orthrus_matrix *y, int32_t rows, int32_t width, void *stream);

/* Weights in the layout that the products read, made once by orthrus_linear_pack: `groups` matrices
 * [n][k] (group-major), or pairs of them (gated: one that the activation is applied to, one that it
 * multiplies).  packed: device, 256-byte aligned, orthrus_linear_packed_bytes(). */
typedef struct orthrus_linear_weights {
    const void *packed;
    int32_t dtype;      /* ORTHRUS_BF16 or ORTHRUS_MX8 */
    int32_t n, k, gated, groups;
} orthrus_linear_weights;

/* Bytes of packed weights (`packed` is not looked at; 0 for invalid sizes, k > 2^22 and n > 2^26). */
size_t orthrus_linear_packed_bytes(const orthrus_linear_weights *w);

/* Writes w->packed from [groups * n][k] matrices of w->dtype (`up` for gated weights, else NULL).  Any strides and
 * alignment to an element; packed shares no byte with them (EINVAL). */
int orthrus_linear_pack(const orthrus_linear_weights *w, const orthrus_matrix *matrix, const orthrus_matrix *up, void *stream);

/* What follows a product.  bias: fp32 device [groups][n] ([groups][2][n] for gated weights: those of the
 * activated matrix, then of the other), or NULL.  residual (data NULL: none): F32 or BF16 rows, added
 * last; may be y itself (data, stride and dtype), else y and the workspace share no byte with anything (EINVAL). */
typedef struct orthrus_epilogue {
    const float *bias;
    int32_t act;
    orthrus_matrix residual;
} orthrus_epilogue;

/* Device workspace bytes that hold what a product of up to `rows` rows may need (the same bound serves every smaller
 * number of rows; at most 64 MiB; 0: none is needed, or invalid arguments). */
size_t orthrus_linear_bytes(const orthrus_linear_weights *w, int32_t rows);

/* y[r] = act(x[r] W^T + bias) + residual[r], or for gated weights act(x W^T + bias) * (x U^T + bias_u) +
 * residual; w->groups is 1.  x: rows of k elements of the weights' type; 16-byte aligned, row stride a multiple of 16
 * bytes; for MX8 scales 4-byte aligned, scale_stride a multiple of 4.  The 16 bytes, of scales the 4, that hold a row's last
 * elements are read whole, what lies between rows may be read, and nothing outside of these is.  y: rows of n elements, F32, BF16 or
 * MX8, any stride and alignment to an element.  epilogue NULL: none.
 *
 * Sums in fp32, in an order that depends on the sizes alone; bf16 products are exact.  The matrix cores add 8-bit products eight
 * neighbours at a time, without the bits below 2^-13 of the power of two of the largest of the eight: 1.5e-5 of a sum of normal data.  Where
 * that counts, blocks that orthrus_convert reads back to BF16 go through weights packed in BF16, exactly, at half the rate.
 *
 * workspace: 16-byte aligned, one call in flight; calls may be captured into graphs.  EINVAL: null pointers, sizes, strides or
 * alignments against the above, memory that is shared; EUNSUPPORTED: types without a kernel; ECAPACITY: workspace too small; k > 2^22,
 * n > 2^26 or rows >= 2^30; 2^31 bytes or more in 256 rows of x or of its scales; more tiles than a launch holds (2^24 of 64 rows by 128
 * weight rows or more; 2^23 of 16 by 16 or more where a group's share is at most 16 rows).  rows = 0 is a no-op. */
int orthrus_linear(const orthrus_linear_weights *w, const orthrus_matrix *x, int32_t rows, const orthrus_epilogue *epilogue,
                   const orthrus_matrix *y, void *workspace, size_t ws_bytes, void *stream);

/* The same for groups of rows: row r of [offsets[g], offsets[g + 1]) goes through the weights and bias of group
 * g.  offsets: int32 device [groups + 1], ascending (a value outside [0, rows] counts as the nearer
 * end, one below an earlier one as the earlier one); groups may be empty.  Rows of y before the first offset and
 * from the last one on are left as they were. */
int orthrus_linear_grouped(const orthrus_linear_weights *w, const orthrus_matrix *x, const int32_t *offsets, int32_t rows,
                           const orthrus_epilogue *epilogue, const orthrus_matrix *y, void *workspace, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ORTHRUS_LINEAR_H */
