/*
 * cc_layers.h -- C ABI of operators of the scoring model (libccjoin.so, next to cc_join.h).
 *
 * The join writes the rows that the scoring model reads; the operators here are those that meet such
 * rows first (Connected Content Retriever, §4): the dense product W h + b with ReLU, and dropout, of
 * a block Dropout(LN(ReLU(W h + b))) of Eq. 2 (its layer norm is not here), and tables of learned
 * rows looked up by id. Eq. 3's table is one of these: S_max + 1 rows of 3 columns, of which
 * E_pos(min(slot, S_max)) is added to the model's 3 logits.
 *
 *   training   cc_embedding_lookup (with dropout), cc_embedding_grad, cc_dropout (forward, and on
 *              the output's gradient the backward pass)
 *   serving    cc_embedding_lookup, cc_quantize_rows, cc_matmul_i8, cc_linear_i8
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

#ifdef __cplusplus
}
#endif

#endif /* CC_LAYERS_H */
