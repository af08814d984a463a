/*
 * tagore_embed.h — C boundary of the operators that learn and serve the vectors a graph is built over.
 *
 * The rows that tg_knn_build indexes are the rows of a table that a model has learnt: ids are looked up in
 * it, the looked-up rows go through a root-mean-square norm with the residual's addition, and a softmax
 * cross entropy over all rows of a table says how well they point at the right one; its gradients lead
 * back to the table.  To serve them, normed rows are put on an 8-bit grid with a scale per row, and scored
 * by an integer product.
 *
 * The conventions are those of tagore_knn.h: pointers are HIP device memory of the current device, owned by
 * the caller; work is only enqueued, on `stream`; nothing is allocated, no call waits for the device, and
 * all of them can be captured into a HIP graph; the return value is a tg_status, tg_last_error() says
 * what was wrong, and outputs are untouched on TG_ERR_INVALID_ARG.  Where a call takes a workspace its
 * size comes from the function of the same name with _workspace (0: the arguments are invalid, or none is needed; then NULL will
 * do); it must be 256-byte aligned and belongs to the call until `stream` has got past it.
 *
 * dtype: a tg_dtype.  Matrices are row-major; `ld` is the distance of two rows in elements, at least
 * the row length (a matrix without `ld` has its rows back to back); rows need no alignment beyond their
 * element's, 16-byte aligned ones are faster.  Sums, norms and softmax statistics are held in 32 bits or
 * more, results are rounded once (the softmax's gradient rounds an intermediate as well, see there).  Equal
 * inputs give equal results, bit for bit: no sum depends on the order in which workgroups arrive.
 */
#ifndef TAGORE_EMBED_H
#define TAGORE_EMBED_H

#include "tagore_knn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { TG_DTYPE_F32 = 0, TG_DTYPE_BF16 = 1, TG_DTYPE_F16 = 2 } tg_dtype;

/*
 * out[t] = scale * table[ids[t]], t = 0..n-1.  table: n_rows x d, ids: n whole numbers of 32 bits, or of 64
 * where ids64 is 1; an id outside [0, n_rows) is no row: its out row is zero.  out: n x d of the table's
 * type.  0 <= n < 2^30, 1 <= n_rows < 2^30, 1 <= d <= 65536.
 */
int tg_embed_lookup(const void* table, int64_t ld, int32_t dtype, int64_t n_rows, int32_t d, const void* ids,
                    int32_t ids64, int64_t n, float scale, void* out, void* stream);

/*
 * The gradient of tg_embed_lookup with respect to the table: row v of out is scale times the sum of grad[t]
 * over the t with ids[t] = v, in fp32 and in an order that depends on the ids alone (the tokens are sorted by
 * id first).  grad: n x d of type dtype.  out: n_rows x d of type out_dtype (TG_DTYPE_F32, or dtype).
 * accumulate = 0: rows without a token become zero; 1: the sums are added to what out holds, and rows
 * without a token are not touched (a table that is also the softmax's: its gradient first, then this; with out in fp32 only the first of
 * the two is rounded to the table's type).
 */
size_t tg_embed_lookup_grad_workspace(int64_t n, int64_t n_rows, int32_t d);
int tg_embed_lookup_grad(const void* grad, int64_t ld, int32_t dtype, const void* ids, int32_t ids64, int64_t n,
                         int64_t n_rows, int32_t d, float scale, int32_t accumulate, void* out, int32_t out_dtype,
                         void* workspace, size_t workspace_bytes, void* stream);

/*
 * r = x + residual, rounded to the type of x (residual = NULL: r = x, and out_r is not written and may be
 * NULL); rstd = 1 / sqrt(mean(r^2) + eps), of whatever size the row is (a row of zeros with eps = 0: infinite, and
 * out_y NaN); out_y = r * rstd * weight.  x, residual: n x d of type dtype; weight: d of the same type; out_y, out_r:
 * n x d; out_rstd: n fp32, or NULL.  out_r may be x or residual itself where that one's rows are back to back (refused
 * otherwise: rows still to be read would be written over).  0 <= n < 2^30, 1 <= d <= 8192, eps >= 0.
 */
int tg_add_rms_norm(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, const void* weight,
                    int32_t dtype, int64_t n, int32_t d, float eps, void* out_y, void* out_r, float* out_rstd,
                    void* stream);

/*
 * The gradient of tg_add_rms_norm: dy is the gradient of out_y, dr (or NULL) that of out_r on its other
 * uses.  out_dx: the gradient of x and of residual alike; out_dweight: d values of type dtype.
 */
size_t tg_add_rms_norm_grad_workspace(int64_t n, int32_t d);
int tg_add_rms_norm_grad(const void* dy, int64_t ld_dy, const void* dr, int64_t ld_dr, const void* r, int64_t ld_r,
                         const void* weight, const float* rstd, int32_t dtype, int64_t n, int32_t d, void* out_dx,
                         void* out_dweight, void* workspace, size_t workspace_bytes, void* stream);

/*
 * tg_add_rms_norm with the normed rows on an 8-bit grid: scale = max|y| / 127 (rounded to fp32) and
 * q = y / scale rounded to the nearest whole number (ties to the even one), -127..127.  out_q: n x d int8,
 * out_scale: n fp32.  A row of zeros has scale 0 (with eps = 0 its norm is not finite); a row that holds a NaN, or whose norm is not finite,
 * has scale NaN and zeros.  y is formed and divided in 64 bits: which side of a border a value falls on does not depend
 * on how the row was cut up.
 */
int tg_add_rms_norm_q8(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, const void* weight,
                       int32_t dtype, int64_t n, int32_t d, float eps, int8_t* out_q, float* out_scale, void* out_r,
                       void* stream);
/* Rows on the same grid without a norm: scale = max|x| / 127. */
int tg_quantize_rows(const void* x, int64_t ld_x, int32_t dtype, int64_t n, int32_t d, int8_t* out_q,
                     float* out_scale, void* stream);
/* What they stand for: out = q * scale, rounded to dtype. */
int tg_dequantize_rows(const int8_t* q, const float* scale, int64_t n, int32_t d, int32_t dtype, void* out, void* stream);

/*
 * out[i][j] = a_scale[i] * b_scale[j] * sum_k a[i][k] b[j][k] (+ bias[j]): a product of 8-bit rows with a
 * scale per token (row of a) and per channel (row of b); the sum is a whole number of 32 bits and exact.
 * a: m x k int8, b: n x k int8 (a weight of n output channels, or the rows of an index), bias: n fp32 or
 * NULL, out: m x n of type dtype.  0 <= m < 2^30, 1 <= n < 2^30, 1 <= k <= 65536 (127 * 128 * k stays below 2^31 for
 * every int8 value).  Beyond 64 tokens and 256 bytes a row, rows
 * whose length or start is no multiple of 16 bytes are copied into the workspace first.  aligned: 1 where a and b
 * both start at a multiple of 16 bytes, 0 where that is not known.
 */
size_t tg_matmul_q8_workspace(int64_t m, int64_t n, int32_t k, int32_t aligned);
int tg_matmul_q8(const int8_t* a, const float* a_scale, const int8_t* b, const float* b_scale, const float* bias,
                 int64_t m, int64_t n, int32_t k, void* out, int32_t dtype, void* workspace, size_t workspace_bytes,
                 void* stream);

/*
 * Softmax cross entropy of n rows against all n_rows rows of a table, without the n x n_rows logits:
 *   z[t][v] = scale * <h[t], w[v]>,  lse[t] = log sum_v exp(z[t][v]),  loss[t] = lse[t] - z[t][targets[t]].
 * A target outside [0, n_rows) is none: the token's loss is 0 and it has no part in any gradient.
 * Infinite logits count as the formulas have them (lse is then infinite, and undefined what takes an infinite one's difference from
 * it); a NaN among a token's logits makes lse NaN, and the loss if it has a target.
 * h: n x d, w: n_rows x d, both of type dtype; targets: n whole numbers of 32 bits, or of 64 where targets64 is 1;
 * out_loss, out_lse: n fp32.  0 <= n < 2^28, 1 <= n_rows < 2^30, 1 <= d <= 8192.
 * Rows are read where they are if they start at a multiple of 16 bytes, are a multiple of 16 bytes (of at most 1 MiB) apart and have
 * such a length; h or w is copied into the workspace first if not (the gradient always copies h).  aligned: of which operand the first two are known:
 * 1 of both, 2 of w, 3 of h, 0 of none.
 */
size_t tg_softmax_xent_workspace(int64_t n, int64_t n_rows, int32_t d, int32_t dtype, int32_t aligned);
int tg_softmax_xent(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int32_t dtype, int64_t n,
                    int64_t n_rows, int32_t d, const void* targets, int32_t targets64, float scale, float* out_loss,
                    float* out_lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Its gradients: with P[t][v] = scale * dloss[t] * (exp(z[t][v] - lse[t]) - [v = targets[t]]),
 * out_dh = P w (n x d) and out_dw = P^T h (n_rows x d), both of type dtype.  lse: what tg_softmax_xent gave, dloss: n
 * fp32, the gradient of every token's loss.  The table is taken in pieces, for each of which P is formed
 * (from the logits, computed again) in the type of the inputs and multiplied twice; a larger workspace than asked for makes larger pieces.
 * So in 16 bits an entry of P is off by up to half a step of the type, except at a token's target, where what was rounded off is given back to
 * both gradients; the result's own rounding comes on top.  In fp16 the P of all tokens is kept under one power of two: entries
 * below 2^-27 of the largest |scale dloss| have steps of 2^-37 of it.
 */
size_t tg_softmax_xent_grad_workspace(int64_t n, int64_t n_rows, int32_t d, int32_t dtype, int32_t aligned);
int tg_softmax_xent_grad(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int32_t dtype, int64_t n,
                         int64_t n_rows, int32_t d, const void* targets, int32_t targets64, const float* lse,
                         const float* dloss, float scale, void* out_dh, void* out_dw, void* workspace,
                         size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TAGORE_EMBED_H */
