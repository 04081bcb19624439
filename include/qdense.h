/*
 * qdense — what stands beside attention and the experts in a layer of a served model, on AMD MI355X (gfx950): the residual's
 * addition with the norm, and products with dense matrices of 4-bit weights (projections, dense feed-forward layers, the
 * vocabulary).  With qattn.h and qmoe.h a layer is
 *
 *     dense_norm -> dense_linear (q, k, v) -> attention -> dense_linear -> dense_norm -> moe_route .. moe_combine
 *
 * each dense_norm adding what the block before it gave to the residual stream.
 *
 * Conventions that hold for every call
 *  - Pointers marked [device] are GPU global memory owned by the caller; the library allocates nothing, creates no stream, keeps
 *    no state between calls and never waits: calls enqueue on `stream` (a hipStream_t as void*, NULL = the default stream) and
 *    return, so they can be captured into a graph.  The current device is that of the pointers and of the stream.
 *  - Return value: MOE_OK or a negative moe_status (qmoe.h), with the text in moe_last_error().  On an error nothing was enqueued
 *    (MOE_E_HIP excepted).
 *  - A call of no tokens does nothing and looks at no pointer of its rows.
 *  - A call's results are the same bits every time.  dense_norm: a row's are the same whatever stands beside it.  dense_linear: a
 *    token's may differ in the last bits with the number of tokens in its call, by which the order of its sums goes.
 *  - A value that is not finite spoils its own row: of dense_norm the row (or head) it stands in, of dense_linear its token.
 */
#ifndef QDENSE_H
#define QDENSE_H

#include "qmoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows: element d of head h of token t is data[t * token_stride + h * head_stride + d].  data 16-byte aligned; strides in elements, not negative,
 * and multiples of 16 bytes (dense_linear's output: any stride, data aligned to its elements).  Rows of an input may share
 * memory (a stride of 0), rows of an output are apart.
 * DENSE_FP8: e4m3 (OCP: largest 448) with one scale byte e8m0 (2^(byte-127)) for every 32 elements of a row, scale
 * [n_tokens, heads, dim/32] dense: value = element * scale.  NULL for the other types. */
enum { DENSE_BF16 = 0, DENSE_F32 = 1, DENSE_FP8 = 2 };
typedef struct {
    void *data;     /* [device] */
    uint8_t *scale; /* [device] */
    int64_t token_stride;
    int64_t head_stride;
    int32_t type;
} dense_rows;

/* Residual and norm.  For each of the n_tokens * heads rows of dim elements
 *     r = x + add      (rounded to add's type; r = x where add is NULL)
 *     total = r
 *     out = r / sqrt(mean(r^2) + eps) * (weight + shift)
 * Sums, means and products are fp32; out is rounded once.  heads is 1 for the norm of whole tokens; with more, each head of a
 * token is normalised by itself (queries and keys, as slices of one product's rows).
 * x: bf16.  add: bf16 or fp32, or NULL.  total: rows of add's type, or NULL; needs add.  out: bf16 or fp8.  weight [device]
 * [dim], 16-byte aligned, of weight_type bf16 or fp32; NULL: 1 (and shift is not looked at).  shift: 1 for weights that are kept
 * as differences from 1, else 0.  eps > 0.  dim: a multiple of 8 (32 for an fp8 out), at most 32768; n_tokens * heads: at most 2^30.
 * total may be add, and out may be x or add, where types and strides are the same; otherwise outputs overlap neither inputs nor each other (rows that
 * begin at the same address are refused, other overlaps are the caller's to avoid).
 * fp8: the scale of 32 elements is the smallest power of two, 2^-126 at least, for which none is over 448 (one that would round
 * to 2^128 to 1.875 * 2^127); each element is rounded once.  32 elements of which one is not finite have the scale byte 255 (NaN).
 * Rows whose sum of squares is over the largest fp32 give zeros (elements of 2^63 and more). */
int32_t dense_norm(const dense_rows *x, const dense_rows *add, const dense_rows *total, const dense_rows *out, const void *weight,
                   int32_t weight_type, float shift, float eps, int32_t n_tokens, int32_t heads, int32_t dim, void *stream);

/* A matrix of 4-bit weights: rows outputs, cols inputs (a multiple of 32), in the microscaling format of qmoe.h: elements e2m1,
 * one scale byte e8m0 for every 32 along a row.  codes and scales are what dense_pack4 wrote: tiles of 16 rows by 128 columns,
 * rows and columns behind the matrix's last zero, tile (r/16, k/128) at ((r/16) * ceil(cols/128) + k/128) * 1024 bytes; in it
 * 16 bytes at ((k%128)/32 * 16 + r%16) * 16, the 32 elements of row r from column k - k%32 on, the one of the lower column in the low nibble.
 * Scales: for each 16 rows by 512 columns 256 bytes, at ((r/16) * ceil(cols/512) + k/512) * 256; in it the byte of row r and columns
 * k - k%32 .. at ((k%128)/32 * 16 + r%16) * 4 + (k%512)/128. */
typedef struct {
    const void *codes;     /* [device] dense_matrix4_code_bytes(rows, cols), 16-byte aligned  */
    const uint8_t *scales; /* [device] dense_matrix4_scale_bytes(rows, cols), 16-byte aligned */
    int32_t rows, cols;
} dense_matrix4;

/* Sizes of a packed matrix; 0 if rows (1 .. 2^24) or cols (a multiple of 32, 32 .. 2^20) is out of range. */
size_t dense_matrix4_code_bytes(int32_t rows, int32_t cols);
size_t dense_matrix4_scale_bytes(int32_t rows, int32_t cols);

/* Packs codes [rows, cols/2] (the element of the even column in the low nibble) and scales [rows, cols/32], both [device] and dense, codes
 * 16-byte aligned, into w's memory; once, when a model is loaded.  w's memory overlaps neither. */
int32_t dense_pack4(const uint8_t *codes, const uint8_t *scales, const dense_matrix4 *w, void *stream);

/* out[t, r] = sum_c x[t, c] w[r, c], x: bf16 or fp8 [n_tokens, cols], out: bf16 or fp32 [n_tokens, rows] (heads is 1; head strides
 * are not looked at).  Sums are fp32, out is rounded once.  Where x is bf16, weights become bf16 operands: exactly, for every scale byte, but for those of 2^128 and more (elements
 * of 4 and 6 with scale byte 253, of 2 to 6 with 254), which are infinite.  fp8 rows with a bf16 out are multiplied as they are, with weights as they are,
 * by the matrix unit's scaled products, which drop, of the few neighbouring products that they add first, what is below 2^-14 of
 * the largest (measured: of normally distributed rows 2^-18 of a result, 2^-14 with large outliers); with an fp32 out both become bf16
 * operands: the rows' elements exactly from 2^-133 on (smaller parts, which scale bytes 0 to 2 alone have, are rounded to multiples of it), infinite from 2^128 on (scale bytes from
 * 247 on; none that dense_norm writes).
 * n_tokens: at most 2^24.  out overlaps no input, the workspace neither.
 * workspace ([device], 16-byte aligned, may be NULL; its contents before and after the call are of no account): where rows are so few that
 * they leave CUs idle, the sums are cut into ranges of columns that run side by side, and a second launch adds them in order.
 * dense_linear_workspace_bytes(...) is what that takes, at most 256 MB, 0 where nothing is cut; with less than that nothing is cut either. */
size_t dense_linear_workspace_bytes(int32_t n_tokens, int32_t rows, int32_t cols, int32_t x_type, int32_t out_type);
int32_t dense_linear(const dense_rows *x, const dense_matrix4 *w, const dense_rows *out, int32_t n_tokens, void *workspace,
                     size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* QDENSE_H */
