/*
 * tagore_learn.h — C boundary of the operators that tune a learnt table by what it answers with.
 *
 * tagore_embed.h says how far a table is from its targets.  Here it is asked how likely given rows are, how sure it is (the
 * entropy), and which rows it would rather have answered with; tuning by rewards takes the gradients of the first two.  In front of the
 * update the gradients of all tensors are brought under one norm.
 *
 * The conventions are those of tagore_embed.h: device memory of the current device, work only enqueued on `stream`, nothing
 * allocated, everything capturable into a HIP graph; a tg_status is returned, and outputs are untouched on TG_ERR_INVALID_ARG.
 * dtype, ld, the workspaces and `aligned` are as there.  Equal inputs give equal results, bit for bit.
 */
#ifndef TAGORE_LEARN_H
#define TAGORE_LEARN_H

#include "tagore_embed.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * For n rows h against all n_rows rows of a table w, without the n x n_rows logits:
 *   z[t][v] = scale * <h[t], w[v]>,  out_lse[t] = log sum_v exp(z[t][v]),  p = exp(z - lse),
 *   out_logp[t] = z[t][targets[t]] - lse[t],  out_entropy[t] = - sum_v p[t][v] log p[t][v],
 * and the `top` best rows: out_rows (n x top) those of the largest z, in that order, and out_row_logp (n x top) their z - lse.  Which rows these
 * are and their order is decided by z in 64 bits, equal ones by the lower row; where the table has fewer rows than top, the rest is
 * row -1 of log probability -infinity.  (All rows whose logits fp32 cannot tell from the last best one's are scored in 64 bits: where these are thousands,
 * as in a table of equal rows, that is what a call takes.  What it can tell goes by |scale| |h| d 2^-22 and the length of the longest of some 64 to 256 neighbours in the table: rows far longer
 * than the others, a thousand times and more, take their neighbours with them, but no others.)  0 <= top <= 32; with 0, out_rows and out_row_logp may be NULL.
 * A target outside [0, n_rows) is none: the token's logp is 0, its other results are as for any other.  targets = NULL: no token has one; out_logp
 * may then be NULL too.  Log probabilities are at most 0: where lse's rounding leaves more, 0 is given.
 * A NaN among a token's logits makes all its results NaN, and its best rows -1.  Infinite logits count as the formulas have them: lse is then infinite, the
 * entropy undefined (NaN), and undefined what takes an infinite logit's difference from it; the best rows are those of the largest logits still.
 * h: n x d, w: n_rows x d, both of type dtype; targets: n whole numbers of 32 bits, or of 64 where targets64 is 1; out_logp,
 * out_entropy, out_lse: n fp32; out_rows: 32 bits; out_row_logp: fp32.  0 <= n < 2^28, 1 <= n_rows < 2^30, 1 <= d <= 8192.
 */
size_t tg_log_probs_workspace(int64_t n, int64_t n_rows, int32_t d, int32_t dtype, int32_t top, int32_t aligned);
int tg_log_probs(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int32_t dtype, int64_t n, int64_t n_rows, int32_t d,
                 const void* targets, int32_t targets64, float scale, int32_t top, float* out_logp, float* out_entropy,
                 float* out_lse, int32_t* out_rows, float* out_row_logp, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The gradients of logp and entropy: with
 *   P[t][v] = scale * (dlogp[t] ([v = targets[t]] - p[t][v]) - dentropy[t] p[t][v] (z[t][v] - lse[t] + entropy[t])),
 * out_dh = P w (n x d) and out_dw = P^T h (n_rows x d), both of type dtype; out_dw = NULL: the table is not learnt, and its gradient not formed.
 * lse, entropy: what tg_log_probs gave; dlogp, dentropy: n fp32; dentropy = NULL: the entropy has no part (then entropy may be NULL).
 * A token without a target has no part through logp, and one without a target whose dentropy is 0 none at all, whatever its logits are.
 * How P is formed, rounded and held is as for tg_softmax_xent_grad.  table: 1 where out_dw is given, 0 where it is NULL: either has a workspace of its own size, and the one
 * without the table's gradient can be the larger (dh comes in up to 64 parts of n x d fp32, which alone are to fill the device).
 */
size_t tg_log_probs_grad_workspace(int64_t n, int64_t n_rows, int32_t d, int32_t dtype, int32_t table, int32_t aligned);
int tg_log_probs_grad(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int32_t dtype, int64_t n, int64_t n_rows, int32_t d,
                      const void* targets, int32_t targets64, const float* lse, const float* dlogp, const float* entropy,
                      const float* dentropy, float scale, void* out_dh, void* out_dw, void* workspace, size_t workspace_bytes,
                      void* stream);

/*
 * The norm of many gradients together: out_norm = |scale| sqrt(sum of the squares of all values of all tensors), fp32, the sum in 64 bits.
 * grads, counts, dtypes: host arrays of `tensors` device pointers, counts of values (back to back in memory) and types; they are read
 * before the call returns.  scale: what the gradients are to be multiplied with (1 over a loss scale).  0 <= tensors <= 2^20,
 * 0 <= counts < 2^40 (a tensor of none may be NULL).
 */
size_t tg_grad_norm_workspace(const int64_t* counts, int32_t tensors);
int tg_grad_norm(const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t tensors, float scale, float* out_norm,
                 void* workspace, size_t workspace_bytes, void* stream);

/*
 * out = grads * scale * min(1, max_norm / norm).  The norm of the factor is the one in 64 bits: where finite values have a norm beyond fp32, out_norm, which is rounded as
 * tg_grad_norm's is, holds infinity, and they are brought under max_norm all the same.  Where a value is infinite or NaN (out_norm then is, too), or the norm is not above max_norm,
 * out = grads * scale.  out: host array of as many device pointers, of tensors of the gradients' counts and types, each its own gradient or memory that no other
 * tensor of the call has a part in (refused otherwise).  max_norm >= 0; infinity: the scale alone.
 * Results are rounded once to their type, behind the product in 32 bits; a gradient in its own place is not written where its factor is 1.
 */
int tg_clip_grads(const void* const* grads, void* const* out, const int64_t* counts, const int32_t* dtypes, int32_t tensors,
                  float max_norm, float scale, float* out_norm, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TAGORE_LEARN_H */
