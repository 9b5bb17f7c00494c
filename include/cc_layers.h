/*
 * cc_layers.h -- C ABI of operators of the scoring model (libccjoin.so, next to cc_join.h).
 *
 * The join writes the rows that the scoring model reads; the operators here are those that meet such
 * rows first (Connected Content Retriever, §4): a block Dropout(LN(ReLU(W h + b))) of Eq. 2 as the
 * dense product with ReLU, the norms before and after a block with its gate and residual sum, and
 * dropout; and tables of learned rows looked up by id. Eq. 3's table is one of these: S_max + 1 rows
 * of 3 columns, of which E_pos(min(slot, S_max)) is added to the model's 3 logits.
 *
 *   training   cc_embedding_lookup (with dropout), cc_embedding_grad, cc_dropout (forward, and on
 *              the output's gradient the backward pass), cc_block_norm, cc_block_norm_grad
 *   serving    cc_embedding_lookup, cc_block_norm; in 8 bits cc_quantize_rows, cc_matmul_i8,
 *              cc_linear_i8; in 4 bits cc_quantize_mxfp4, cc_dequantize_mxfp4, cc_matmul_mxfp4,
 *              cc_linear_mxfp4
 *
 * Conventions are those of cc_join.h: caller-owned device memory, work enqueued on `stream`, no
 * synchronisation, no allocation, nothing enqueued after an argument error, no exception across
 * the interface. Calls run on the current HIP device. They may be captured into a HIP graph; a
 * replay uses the captured scalars (of dropout: the same mask). In addition:
 *   - Matrices are rows of dense elements with a row stride in bytes, which is a multiple of the
 *     element size and at least the row's width (ignored when there are fewer than two rows).
 *     Pointers are aligned to their element size unless stated otherwise. 16-byte alignment of
 *     pointers and strides is faster.
 *   - An output must not overlap an input or the workspace (CC_ERR_INVALID_ARGUMENT), except
 *     where in-place use is stated. A matrix counts from its first element to its last: side by side
 *     in one buffer's rows, two matrices overlap.
 *   - A workspace is device scratch, 16-byte aligned, whose contents need no preparation and are
 *     not kept from one call to the next; two calls that may run at the same time need one each.
 *   - A call with no output elements returns CC_OK and enqueues nothing.
 */
#ifndef CC_LAYERS_H
#define CC_LAYERS_H

#include "cc_join.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. Arithmetic is in 32 bits for all of them, rounded once (to nearest even) when a
 * result is stored. */
#define CC_F32 0
#define CC_F16 1
#define CC_BF16 2

/*
 * Dropout's mask. It is a function of (seed, site, row, column) and never stored: the backward
 * pass, a recomputation or another rank draws it again.
 *
 *   T = 65536 - floor(65536 p + 1/2), so p acts rounded to the nearest multiple of 2^-16.
 *   Element (row, column) is kept iff its 16 bits are below T, and scaled by 65536 / T.
 *   Its 16 bits are number column % 8 of the words x0..x3 (low half of a word first) of
 *   Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3",
 *   SC 2011) at counter (row mod 2^32, row / 2^32, column / 8, site), key (seed mod 2^32,
 *   seed / 2^32).
 *
 *   p          probability of dropping an element, in [0, 1]; 0 keeps everything unscaled, 1
 *              drops everything.
 *   seed       64 bits; one per step, for example.
 *   site       which of the program's dropouts this is: masks of different sites or seeds are
 *              independent.
 *   first_row  number of the call's first row, >= 0, first_row + rows < 2^63: a shard or a
 *              micro-batch of a larger batch draws its part of the whole batch's mask.
 *
 * A dropped element contributes nothing, whatever its value: a NaN or an infinity there does not
 * reach the result.
 */

/*
 * cc_embedding_lookup -- rows of a table by id, scaled, with an optional dropout.
 *
 *   out[t][c] = keep(first_row + t, c) ? table[ids[t]][c] * (scale * 65536 / T) : 0
 *
 * An id outside [0, n_rows) gives a zero row (the -1 of §6.3.1, Eq. 6: not found; also a padding
 * id).
 *
 *   table       [n_rows][cols] of table_type, row stride table_stride bytes.
 *   ids         [n_ids], id_bytes = 8 (int64) or 4 (int32).
 *   cols        elements per row, 1 to 2^24.
 *   scale       factor, rounded to 32 bits together with 65536 / T.
 *   out         [n_ids][cols] of out_type, row stride out_stride bytes. out_type is table_type, or
 *               CC_F16 or CC_BF16 for a table in CC_F32.
 * Errors: CC_ERR_INVALID_ARGUMENT, CC_ERR_DEVICE.
 */
CC_API cc_status cc_embedding_lookup(const void *table, int64_t n_rows, int64_t table_stride,
                                     int32_t table_type, const void *ids, int32_t id_bytes,
                                     int64_t n_ids, int32_t cols, double scale, double p,
                                     uint64_t seed, uint32_t site, int64_t first_row, void *out,
                                     int64_t out_stride, int32_t out_type, hipStream_t stream);

/*
 * cc_embedding_grad -- gradient of cc_embedding_lookup with respect to its table.
 *
 *   grad_table[r][c] = (scale * 65536 / T) * sum of grad_out[t][c] over the t with ids[t] = r and
 *                      keep(first_row + t, c)   [ + grad_table[r][c] if accumulate ]
 *
 * The ids are sorted (stably) and each row's gradients are summed in 32 bits in an order that
 * depends on the call's sizes and ids alone, so that equal calls give equal bits; no atomic
 * operation touches a value. Ids outside [0, n_rows) take part in no row.
 *
 *   ids, id_bytes, cols, scale, p, seed, site, first_row   those of the forward call.
 *   n_ids       0 to 2^31 - 1.
 *   grad_out    [n_ids][cols] of grad_type, row stride grad_out_stride bytes.
 *   n_rows      rows of the table, 0 to 2^31 - 2.
 *   grad_table  [n_rows][cols] of table_type, row stride grad_table_stride bytes: CC_F32 or
 *               grad_type. Without accumulate every row is written (zeros where no id points);
 *               with it only rows that an id points at are, each sum rounded once.
 *   workspace   cc_embedding_grad_workspace_bytes(n_ids, n_rows, cols) bytes.
 * Errors: CC_ERR_INVALID_ARGUMENT, CC_ERR_DEVICE.
 */
CC_API int64_t cc_embedding_grad_workspace_bytes(int64_t n_ids, int64_t n_rows, int32_t cols);
CC_API cc_status cc_embedding_grad(const void *ids, int32_t id_bytes, int64_t n_ids,
                                   const void *grad_out, int64_t grad_out_stride,
                                   int32_t grad_type, int32_t cols, double scale, double p,
                                   uint64_t seed, uint32_t site, int64_t first_row,
                                   int64_t n_rows, void *grad_table, int64_t grad_table_stride,
                                   int32_t table_type, int32_t accumulate, void *workspace,
                                   int64_t workspace_bytes, hipStream_t stream);

/*
 * cc_dropout -- out = dropout(x) (+ residual).
 *
 *   out[r][c] = (keep(first_row + r, c) ? x[r][c] * (65536 / T) : 0) + residual[r][c]
 *
 * With the gradient of out in x's place and no residual this is the gradient with respect to x;
 * the residual's gradient is that of out unchanged.
 *
 *   x, out      [n_rows][cols] of `type`, row strides in bytes.
 *   residual    the same, or NULL.
 *   cols        1 to 2^24.
 * In place: out may be x, or residual, where pointer and stride are the same.
 * Errors: CC_ERR_INVALID_ARGUMENT, CC_ERR_DEVICE.
 */
CC_API cc_status cc_dropout(const void *x, int64_t x_stride, const void *residual,
                            int64_t residual_stride, int64_t n_rows, int32_t cols, int32_t type,
                            double p, uint64_t seed, uint32_t site, int64_t first_row, void *out,
                            int64_t out_stride, hipStream_t stream);

/*
 * cc_quantize_rows -- 8-bit integers with one scale per row (of activations: per token; of a
 * weight matrix [outputs][inputs]: per output channel).
 *
 *   most = max |x[r][c]| over the row;  scales[r] = most / 127
 *   q[r][c] = x[r][c] * (127 / most), rounded to nearest even: in [-127, 127]
 *
 * A row of zeros has scale 0. A row that holds a NaN or an infinity has scale NaN and q = 0, so
 * that what is computed from it is NaN instead of a plausible number.
 *
 *   x           [n_rows][cols] of `type`, row stride x_stride bytes.
 *   cols        1 to 2^24.
 *   q           [n_rows][padded] int8, row stride q_stride bytes, 16-byte aligned with q_stride a
 *               multiple of 16; padded = cols rounded up to a multiple of 16, and columns cols to
 *               padded - 1 are written as zeros.
 *   scales      [n_rows] float.
 * Errors: CC_ERR_INVALID_ARGUMENT, CC_ERR_DEVICE.
 */
CC_API cc_status cc_quantize_rows(const void *x, int64_t x_stride, int32_t type, int64_t n_rows,
                                  int32_t cols, int8_t *q, int64_t q_stride, float *scales,
                                  hipStream_t stream);

/*
 * cc_matmul_i8 -- product of 8-bit rows with 8-bit weights, a scale for each row of either.
 *
 *   out[i][j] = act((sum_l a[i][l] * b[j][l]) * a_scales[i] * b_scales[j] + bias[j])
 *
 * The sum is exact (32-bit integers); the scales and the bias are applied in 32-bit floating
 * point and the result is rounded once. act is max(., 0) with relu (NaN stays NaN), else identity.
 *
 *   a           [m][k] int8, row stride a_stride bytes; b: [n][k] int8, row stride b_stride bytes
 *               (a linear layer's weights, one row per output). 16-byte aligned, strides and k
 *               multiples of 16, the form that cc_quantize_rows writes (its zero columns add
 *               nothing).
 *   m, n        >= 0, below 2^31 (within 256 of it, a launch has too many workgroups:
 *               CC_ERR_DEVICE).
 *   k           0 to 131,056 (no sum of products of values in [-128, 127] passes 31 bits).
 *   a_scales    [m] float; b_scales: [n] float; bias: [n] float or NULL.
 *   out         [m][n] of out_type, row stride out_stride bytes.
 *   workspace   cc_matmul_i8_workspace_bytes(m, n, k) bytes, NULL where that is 0. No size needs
 *               any now.
 * Errors: CC_ERR_INVALID_ARGUMENT, CC_ERR_DEVICE.
 */
CC_API int64_t cc_matmul_i8_workspace_bytes(int64_t m, int64_t n, int64_t k);
CC_API cc_status cc_matmul_i8(const int8_t *a, int64_t a_stride, const float *a_scales,
                              const int8_t *b, int64_t b_stride, const float *b_scales,
                              const float *bias, int64_t m, int64_t n, int64_t k, int32_t relu,
                              void *out, int64_t out_stride, int32_t out_type, void *workspace,
                              int64_t workspace_bytes, hipStream_t stream);

/*
 * cc_linear_i8 -- cc_quantize_rows of x, then cc_matmul_i8 with weights that are in 8 bits already:
 * a serving layer act(x W' + bias) on floating-point rows, in one call. The quantised rows stay in
 * the workspace or in the kernel; the result is that of the two calls.
 *
 *   x           [m][k] of `type`, row stride x_stride bytes, k >= 1 of any remainder mod 16.
 *   w           [n][padded] int8, row stride w_stride bytes, as cc_quantize_rows writes it from
 *               [n][k] weights (padded = k rounded up to a multiple of 16), w_scales: [n] float.
 *   out         [m][n] of `type`.
 *   workspace   cc_linear_i8_workspace_bytes(m, n, k) bytes.
 * Other arguments as in cc_matmul_i8. Errors: CC_ERR_INVALID_ARGUMENT, CC_ERR_DEVICE.
 */
CC_API int64_t cc_linear_i8_workspace_bytes(int64_t m, int64_t n, int64_t k);
CC_API cc_status cc_linear_i8(const void *x, int64_t x_stride, int32_t type, const int8_t *w,
                              int64_t w_stride, const float *w_scales, const float *bias,
                              int64_t m, int64_t n, int64_t k, int32_t relu, void *out,
                              int64_t out_stride, void *workspace, int64_t workspace_bytes,
                              hipStream_t stream);

/* Norms of a row v of `cols` elements, each followed by "* weight + bias" (1 and 0 where NULL). */
#define CC_NORM_NONE 0  /* v */
#define CC_NORM_RMS 1   /* v / sqrt(mean of v^2 + eps) */
#define CC_NORM_LAYER 2 /* (v - mean) / sqrt(variance + eps), the variance the mean of (v - mean)^2 */

/* What a gate's element u multiplies by. */
#define CC_GATE_LINEAR 0  /* u */
#define CC_GATE_SIGMOID 1 /* 1 / (1 + exp(-u)) */

/*
 * cc_block_norm -- what lies between one block and the next: the norm of a block's output, its gate,
 * the residual sum, and the norm that the next block begins with.
 *
 *   n = post(f);  y[r][c] = x[r][c] + scale * g[r][c] * n[r][c];  h = pre(y)
 *
 * post and pre are norms with a weight and a bias of their own. Without x, y = scale * g * n; without a
 * gate, g = 1; without h, only y is written. A layer norm alone is f, post and y. h is computed from y
 * in 32 bits, not from the rounded y.
 *
 *   x           [n_rows][cols] of stream_type (the residual stream), or NULL.
 *   f           [n_rows][cols] of `type`; gate: the same, or NULL (gate_kind is then ignored).
 *   type        of f, gate and h; stream_type: of x and y, which is `type` or CC_F32.
 *   post_norm, pre_norm    CC_NORM_*; pre_* is ignored without h.
 *   *_weight, *_bias       [cols] float, or NULL.
 *   *_eps       ignored for CC_NORM_NONE; else from 2^-126 up and finite in 32 bits.
 *   scale       finite; rounded to 32 bits.
 *   n_rows      below 2^31; cols: 1 to 2^24.
 *   y           [n_rows][cols] of stream_type; h: [n_rows][cols] of `type`, or NULL.
 * In place: y may be x, and h may be f, where pointer and stride are the same.
 * Squares are summed in 32 bits: rows whose sum of squares passes 3.4e38 are not normalised. Arithmetic
 * is in 32 bits, with approximations of the hardware: inverse roots and reciprocals are within a unit
 * in the last place, and exp(-|u|) of a sigmoid is off by up to |u| + 2 units, so that a gate at u = -80
 * has a relative error of 1e-5. post's weight and bias are multiplied by scale before rows meet them.
 * Errors: CC_ERR_INVALID_ARGUMENT, CC_ERR_DEVICE.
 */
CC_API cc_status cc_block_norm(const void *x, int64_t x_stride, int32_t stream_type, const void *f,
                               int64_t f_stride, const void *gate, int64_t gate_stride,
                               int32_t gate_kind, int32_t type, int32_t post_norm,
                               const float *post_weight, const float *post_bias, double post_eps,
                               int32_t pre_norm, const float *pre_weight, const float *pre_bias,
                               double pre_eps, double scale, int64_t n_rows, int32_t cols, void *y,
                               int64_t y_stride, void *h, int64_t h_stride, hipStream_t stream);

/*
 * cc_block_norm_grad -- gradients of cc_block_norm, from those of y and h.
 *
 * The forward call's x, f and gate are read again and its norms computed again: neither y nor a row's
 * statistics need to be kept. With t = dh * pre_weight, yn the normalised y, Y = dy + (the gradient
 * of pre's norm from t), likewise fn and F = Y * scale * g * post_weight:
 *
 *   dx = Y                                   df = the gradient of post's norm from F
 *   dgate = Y * scale * n * (1, or g (1 - g) for a sigmoid)
 *   d_post_weight = sum over rows of Y * scale * g * fn     d_post_bias = sum of Y * scale * g
 *   d_pre_weight  = sum over rows of dh * yn                d_pre_bias  = sum of dh
 *
 * where the gradient of a norm with factor 1 / s from t is, along each row, t for CC_NORM_NONE,
 * (t - yn mean(t yn)) / s for CC_NORM_RMS and (t - mean(t) - yn mean(t yn)) / s for CC_NORM_LAYER.
 *
 *   x           the forward call's; NULL where that had none, or without dh (it is not read then).
 *   post_bias   the forward call's (dgate depends on it). pre's bias has no part.
 *   dy          [n_rows][cols] of stream_type, or NULL for zeros; dh: [n_rows][cols] of `type`, or NULL
 *               where h was not written or not used. One of the two is given.
 *   dx          [n_rows][cols] of stream_type, or NULL; df: [n_rows][cols] of `type`; dgate: the same,
 *               or NULL (it needs a gate).
 *   d_*         [cols] float, or NULL; d_pre_* need dh. Sums are in 32 bits in an order that
 *               depends on n_rows, cols and whether stream_type is CC_F32: equal calls give equal
 *               bits. With `accumulate` they are added to what is there. A call with no rows
 *               writes zeros (accumulate: nothing).
 *   workspace   cc_block_norm_grad_workspace_bytes(n_rows, cols) bytes.
 * Other arguments as in cc_block_norm. In place: dx may be dy, and df may be dh, where pointer and
 * stride are the same. Errors: CC_ERR_INVALID_ARGUMENT, CC_ERR_DEVICE.
 */
CC_API int64_t cc_block_norm_grad_workspace_bytes(int64_t n_rows, int32_t cols);
CC_API cc_status cc_block_norm_grad(
    const void *x, int64_t x_stride, int32_t stream_type, const void *f, int64_t f_stride,
    const void *gate, int64_t gate_stride, int32_t gate_kind, int32_t type, int32_t post_norm,
    const float *post_weight, const float *post_bias, double post_eps, int32_t pre_norm,
    const float *pre_weight, double pre_eps, double scale, int64_t n_rows, int32_t cols,
    const void *dy, int64_t dy_stride, const void *dh, int64_t dh_stride, void *dx,
    int64_t dx_stride, void *df, int64_t df_stride, void *dgate, int64_t dgate_stride,
    float *d_post_weight, float *d_post_bias, float *d_pre_weight, float *d_pre_bias,
    int32_t accumulate, void *workspace, int64_t workspace_bytes, hipStream_t stream);

/*
 * cc_quantize_mxfp4 -- rows in microscaled 4-bit floating point (OCP Microscaling Formats 1.0: E2M1
 * values, an E8M0 scale for each 32 of a row).
 *
 *   Of a block of 32 columns, s = max(0, e - 2), e the biased exponent of the largest magnitude
 *   rounded to one bit of mantissa (nearest, ties to even); its scale is 2^(s - 127).
 *   A value is x / 2^(s - 127) rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the
 *   even code) with x's sign; beyond 6 it is 6.
 *
 * The largest magnitude of a block lies from 3.5 to 7 scales, so that no value is off by more than half
 * the distance of the grid at it, continued past 6. A block that holds a NaN or an infinity has
 * s = 255 (NaN) and zeros: what is computed from it is NaN.
 *
 *   x           [n_rows][cols] of `type`, row stride x_stride bytes.
 *   n_rows      below 2^31; cols: 1 to 2^24.
 *   q           [n_rows][padded / 2], row stride q_stride bytes, 16-byte aligned with q_stride a
 *               multiple of 16; padded = cols rounded up to a multiple of 128. Two values to a
 *               byte, the first in the low half: a value's code is its sign in bit 3 and its
 *               number in the list above. Columns cols to padded - 1 are zeros.
 *   scales      [n_rows][16 * ceil(cols / 512)], row stride scales_stride bytes, 16-byte aligned
 *               with scales_stride a multiple of 16: s of block i at byte i, zeros behind.
 * Errors: CC_ERR_INVALID_ARGUMENT, CC_ERR_DEVICE.
 */
CC_API cc_status cc_quantize_mxfp4(const void *x, int64_t x_stride, int32_t type, int64_t n_rows,
                                   int32_t cols, uint8_t *q, int64_t q_stride, uint8_t *scales,
                                   int64_t scales_stride, hipStream_t stream);

/*
 * cc_dequantize_mxfp4 -- the values of rows in the form that cc_quantize_mxfp4 writes.
 *
 *   out[r][c] = value of q[r][c] * 2^(scales[r][c / 32] - 127), rounded once; NaN where s is 255.
 *
 *   q, scales   as above; columns from cols on are not read.
 *   out         [n_rows][cols] of out_type, row stride out_stride bytes.
 * Errors: CC_ERR_INVALID_ARGUMENT, CC_ERR_DEVICE.
 */
CC_API cc_status cc_dequantize_mxfp4(const uint8_t *q, int64_t q_stride, const uint8_t *scales,
                                     int64_t scales_stride, int64_t n_rows, int32_t cols, void *out,
                                     int64_t out_stride, int32_t out_type, hipStream_t stream);

/*
 * cc_matmul_mxfp4 -- product of 4-bit rows with 4-bit weights, a scale for each 32 values of either.
 *
 *   out[i][j] = act(sum_l a[i][l] * b[j][l] + bias[j])
 *
 * a and b stand for the values that cc_dequantize_mxfp4 gives. Products are exact, their sum is in 32
 * bits in an order that depends on m, n, k and whether a row stride passes 2^24 bytes: equal calls
 * give equal bits, and a view of rows that lie further apart need not give those of its dense copy.
 * The result is rounded once. act as in cc_matmul_i8.
 *
 *   a           [m][k / 2], row stride a_stride bytes; b: [n][k / 2], row stride b_stride bytes (a
 *               linear layer's weights, one row per output); a_scales: [m][16 * ceil(k / 512)],
 *               b_scales: [n][the same], row strides in bytes: all as cc_quantize_mxfp4 writes
 *               them (its zeros add nothing). Rows of scales are read up to their whole width.
 *   m, n        >= 0, below 2^31 (within 256 of it, a launch has too many workgroups:
 *               CC_ERR_DEVICE).
 *   k           0 to 2^24, a multiple of 128.
 *   bias        [n] float or NULL.
 *   out         [m][n] of out_type, row stride out_stride bytes.
 *   workspace   cc_matmul_mxfp4_workspace_bytes(m, n, k) bytes, NULL where that is 0. No size needs
 *               any now.
 * Errors: CC_ERR_INVALID_ARGUMENT, CC_ERR_DEVICE.
 */
CC_API int64_t cc_matmul_mxfp4_workspace_bytes(int64_t m, int64_t n, int64_t k);
CC_API cc_status cc_matmul_mxfp4(const uint8_t *a, int64_t a_stride, const uint8_t *a_scales,
                                 int64_t a_scales_stride, const uint8_t *b, int64_t b_stride,
                                 const uint8_t *b_scales, int64_t b_scales_stride,
                                 const float *bias, int64_t m, int64_t n, int64_t k, int32_t relu,
                                 void *out, int64_t out_stride, int32_t out_type, void *workspace,
                                 int64_t workspace_bytes, hipStream_t stream);

/*
 * cc_linear_mxfp4 -- cc_quantize_mxfp4 of x, then cc_matmul_mxfp4 with weights that are in 4 bits
 * already: a serving layer act(x W' + bias) on floating-point rows, in one call. It has no gradient.
 * The order of its sums follows the same sizes and is not always cc_matmul_mxfp4's: of few rows the
 * last bits may differ from those of the two calls.
 *
 *   x           [m][k] of `type`, row stride x_stride bytes, k from 1 to 2^24, any remainder.
 *   w, w_scales    [n] rows as cc_quantize_mxfp4 writes them from [n][k] weights.
 *   out         [m][n] of `type`.
 *   workspace   cc_linear_mxfp4_workspace_bytes(m, n, k) bytes.
 * Other arguments as in cc_matmul_mxfp4. Errors: CC_ERR_INVALID_ARGUMENT, CC_ERR_DEVICE.
 */
CC_API int64_t cc_linear_mxfp4_workspace_bytes(int64_t m, int64_t n, int64_t k);
CC_API cc_status cc_linear_mxfp4(const void *x, int64_t x_stride, int32_t type, const uint8_t *w,
                                 int64_t w_stride, const uint8_t *w_scales, int64_t w_scales_stride,
                                 const float *bias, int64_t m, int64_t n, int64_t k, int32_t relu,
                                 void *out, int64_t out_stride, void *workspace,
                                 int64_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* CC_LAYERS_H */
