/*
 * elas_loss.h -- C ABI of the losses of a training step: log-probabilities of
 * tokens from logits with their gradient, and the losses on them (token loss,
 * clipped policy loss, preference loss), each with its gradient in the same call.
 * Part of libelas; the conventions, status codes, debug mode and timing calls of
 * elas.h and elas_train.h hold here too: device pointers owned by the caller,
 * arguments checked on the host before anything is enqueued, everything
 * asynchronous on `stream`, nothing allocated.
 *
 * Shared by the calls on logits, for T tokens over a vocabulary of V:
 *
 * logits   T rows of V values, bf16 (ELAS_LOGITS_F32: float32), row t at logits + t ld;
 *          ld >= V.  Any alignment of the element will do, so rows may have any pitch.
 * ids      [T] int32 (ELAS_IDS_I64: int64).  A token whose id is outside 0 .. V-1
 *          (padding, a prompt) takes no part: its logits are not read, its results
 *          are 0, and its row of the gradient is zeros.
 * scale    z = scale logits (the inverse temperature), 0 < scale <= 2^100.
 * With lse_t = log sum_j exp z_tj, logp_t = z_t,id - lse_t and p = exp(z - lse).
 * dlogits  T rows of V values of the logits' type, row t at dlogits + t ld_out, ld_out >= V;
 *          what lies behind the V values of a row is not touched.  It may be
 *          logits itself with the same pitch (every row is read before it is
 *          written).
 * What a call writes, its workspace included, overlaps nothing else of it but where that is said
 * (ELAS_ERR_OVERLAP); what lies between a row's V values and the next row is not the matrix's.
 * Per-token operands and results are float32 [T] and need 4-byte alignment.
 * Sums over the vocabulary are float32, in groups of at most 32 values, of which a thread adds up at most
 * 16 + V / 8192; per-token terms and sums over tokens are 64-bit.  Their order is fixed by the sizes, the types and the
 * alignment of the rows.
 * A logit may be -inf (its p is 0).  Where a row holds nothing but -inf, a NaN or +inf,
 * its results follow the formulas (NaN, lse -inf), and so do the statistics; other rows do not change.
 * Requires 0 <= T < 2^31, 0 < V <= 2^30.  With T == 0 statistics are zeros and nothing else is
 * written.
 */
#ifndef ELAS_LOSS_H
#define ELAS_LOSS_H

#include "elas_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- flags (with ELAS_IDS_I64 of elas_train.h) ------------------------------ */
/* logits and dlogits are float32 instead of bf16. */
#define ELAS_LOGITS_F32     1u

/*
 * elas_token_logp_fwd -- logp and lse of every token.  lse may be NULL.
 */
int elas_token_logp_fwd(const void* logits, int64_t ld, const void* ids, int64_t T, int64_t V, float scale,
                        uint32_t flags, float* logp, float* lse, void* stream);

/*
 * elas_token_logp_bwd -- gradient of the logits from those of logp and lse:
 *
 *     dlogits_tj = scale (dlogp_t (1[j = id_t] - p_tj) + dlse_t p_tj)
 *
 * lse is that of elas_token_logp_fwd on these logits (of a loss too, where no weight is 0) (p = exp(z - lse) has a relative error of 2^-24 (|z| + 3 |z - lse| + 6);
 * where |lse| is above 64 (bf16 logits: 4096) or not finite the row's sum is taken anew); dlse NULL: zero.
 */
int elas_token_logp_bwd(const float* dlogp, const float* dlse, const void* logits, int64_t ld, const void* ids,
                        const float* lse, int64_t T, int64_t V, float scale, uint32_t flags, void* dlogits,
                        int64_t ld_out, void* stream);

/*
 * elas_token_loss -- cross-entropy of the tokens with weights and a term that
 * keeps lse near 0, and its gradient, from one pass over the logits:
 *
 *     stats[0] = reduce sum_t w_t (-logp_t + z_coef lse_t^2),
 *     stats[1] = reduce sum_t w_t z_coef lse_t^2
 *     dlogits_tj = scale reduce w_t (p_tj - 1[j = id_t] + 2 z_coef lse_t p_tj)
 *
 * weight NULL: 1; a token of weight 0 takes no part.  logp, lse, dlogits may be
 * NULL: not wanted.  stats: device float32 [2].
 * workspace (of this call and the next): 16-byte aligned, at least
 * elas_token_loss_workspace_bytes(T, V, flags) bytes, which is 0 for sizes that no call takes and never less for more tokens.
 */
size_t elas_token_loss_workspace_bytes(int64_t T, int64_t V, uint32_t flags);
int elas_token_loss(const void* logits, int64_t ld, const void* ids, const float* weight, int64_t T, int64_t V,
                    float scale, float reduce, float z_coef, uint32_t flags, float* logp, float* lse, void* dlogits,
                    int64_t ld_out, float* stats, void* workspace, size_t workspace_bytes, void* stream);

/*
 * elas_policy_loss -- the clipped policy loss with a KL term, and its gradient:
 * with r = exp(logp - old_logp), q = ref_logp - logp and advantage A of the token,
 *
 *     l_t  = -min(r A, clamp(r, 1 - clip_low, 1 + clip_high) A),   k_t = exp(q) - q - 1
 *     stats[0] = reduce sum_t w_t (l_t + kl_coef k_t)
 *     stats[1] = reduce sum_t w_t k_t
 *     stats[2] = reduce sum_t w_t [the clamp holds: A > 0, r > 1 + clip_high or A < 0, r < 1 - clip_low]
 *     dlogp_t = reduce w_t (-r A [the clamp does not hold] - kl_coef (exp(q) - 1))
 *     dlogits_tj = scale dlogp_t (1[j = id_t] - p_tj)
 *
 * A coefficient or an advantage of 0 takes no part, as large as what it multiplies may be.
 * old_logp NULL: the policy that sampled the tokens is this one (r = 1, with its
 * gradient).  ref_logp NULL: no KL term (kl_coef is then 0).  weight NULL: 1; a
 * token of weight 0 takes no part.  logp and dlogits may be NULL: not wanted.
 * stats: device float32 [3].  Requires 0 <= clip_low <= 1, clip_high >= 0 (infinite: no upper bound), finite reduce and kl_coef.
 */
int elas_policy_loss(const void* logits, int64_t ld, const void* ids, const float* advantage, const float* old_logp,
                     const float* ref_logp, const float* weight, int64_t T, int64_t V, float scale, float reduce,
                     float clip_low, float clip_high, float kl_coef, uint32_t flags, float* logp, void* dlogits,
                     int64_t ld_out, float* stats, void* workspace, size_t workspace_bytes, void* stream);

/*
 * elas_preference_loss -- the loss of paired answers by their log-ratios, and its
 * gradient.  Sequence s holds the values offsets[s] .. offsets[s+1]-1 of logp; pair
 * i is sequence 2i (chosen) and 2i+1 (rejected).  With c and d their sums of logp
 * - ref_logp,
 *
 *     z_i = beta (c_i - d_i),  l_i = -(1 - smoothing) log sigmoid(z_i) - smoothing log sigmoid(-z_i)
 *     stats = mean_i l_i, share of z_i > 0, mean_i z_i;   margin_i = z_i
 *     dlogp = +-beta (smoothing sigmoid(z_i) - (1 - smoothing) sigmoid(-z_i)) / pairs over the chosen / rejected answer
 *
 * logp, ref_logp [N] float32 (ref_logp NULL: 0); offsets [2 pairs + 1] int32
 * (ELAS_IDS_I64: int64), in rising order; the kernel holds each to 0 .. N.
 * margin [pairs] and dlogp [N] float32 may be NULL; dlogp may be logp; it is 0 in front of the
 * first sequence and behind the last one.  A sequence may be empty (its sum is 0).
 * stats: device float32 [3], zeros where there are no pairs.  Sums are 64-bit, in a fixed order.
 * Requires 0 <= pairs < 2^30, 0 <= N < 2^40, 0 <= smoothing <= 1, finite beta.
 * workspace >= elas_preference_loss_workspace_bytes(N, pairs) bytes (0 for few short answers, and for
 * sizes that no call takes).
 */
size_t elas_preference_loss_workspace_bytes(int64_t N, int64_t pairs);
int elas_preference_loss(const float* logp, const float* ref_logp, const void* offsets, int64_t N, int64_t pairs, float beta,
                         float smoothing, uint32_t flags, float* margin, float* dlogp, float* stats, void* workspace,
                         size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ELAS_LOSS_H */
