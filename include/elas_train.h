/*
 * elas_train.h -- C ABI of the operators around the ELAS FFN in a training
 * step: the norms before and after a block with its gate and residual scale
 * (the pre-norm RMSNorm architecture of Sec. 4.1), the token embedding, and the
 * global norm and clipping of the gradients.  Part of libelas; the conventions,
 * status codes, debug mode and timing calls of elas.h hold here too:
 * device pointers owned by the caller, bf16 as uint16_t bit patterns, dense
 * row-major tensors, 16-byte aligned pointers (except where stated), arguments
 * checked on the host before anything is enqueued, everything asynchronous on
 * `stream`, nothing allocated.  The workspace sizes of sizes that no call takes
 * are 0.
 */
#ifndef ELAS_TRAIN_H
#define ELAS_TRAIN_H

#include "elas.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- flags ---------------------------------------------------------------- */
/* elas_norm_join_*, elas_embed_*: the residual stream (h, h_out, dh_out, dh; x, dx)
   is float32 instead of bf16. */
#define ELAS_RES_F32        1u
/* elas_norm_join_*: the gate holds a row for each token, [T,d], instead of one
   row [d] for all of them. */
#define ELAS_GATE_TOKEN     2u
/* elas_embed_*: ids are int64 instead of int32. */
#define ELAS_IDS_I64        4u
/* elas_embed_bwd: add to dtable instead of overwriting it. */
#define ELAS_EMBED_ADD      8u

/* elas_grad_*: type of a gradient tensor. */
#define ELAS_GRAD_F32       0
#define ELAS_GRAD_BF16      1

/*
 * elas_norm_join_fwd -- joins a block's output to the residual stream and
 * normalises the sum for the next block, in one pass.  For every token t, with
 * i over the d features:
 *
 *     u_i  = b_i w_post_i / sqrt(mean_i b_i^2 + eps)         (w_post NULL: u = b)
 *     h'_i = res_scale h_i + block_scale gate_i u_i          (gate NULL: 1)
 *     n_i  = h'_i w_pre_i / sqrt(mean_i h'_i^2 + eps)
 *
 * h [T,d] residual stream (bf16, or float32 with ELAS_RES_F32); b [T,d] bf16 the
 * block's output; gate bf16, [d] or (ELAS_GATE_TOKEN) [T,d]; w_post, w_pre [d] bf16.
 * Outputs: h_out [T,d] = h' in h's type, n [T,d] bf16.
 * b NULL: there is no block yet, n = norm of h alone (gate, w_post and h_out are
 *   then NULL, both scales unused).
 * w_pre NULL: no norm after the sum (n is then NULL).
 * h_out may be h, and n may be b (each row is read before it is written);
 * otherwise outputs overlap nothing.
 * All arithmetic and both means are float32 (a row of b or h' whose squares leave
 * its range has an infinite mean, or, with eps 0, a mean of 0); h' and n are rounded
 * once, n from the unrounded h'.  A token whose row holds an infinity or NaN affects its own row only.
 * Requires T >= 0, d > 0, d % 8 == 0, d <= 65536, eps >= 0, finite scales.
 * T == 0 is a no-op (pointers are then not inspected and may be NULL).
 */
int elas_norm_join_fwd(const void* h, const uint16_t* b, const uint16_t* gate, const uint16_t* w_post,
                       const uint16_t* w_pre, int64_t T, int64_t d, float res_scale, float block_scale, float eps,
                       uint32_t flags, void* h_out, uint16_t* n, void* stream);

/*
 * elas_norm_join_bwd -- gradient of elas_norm_join_fwd.
 *
 * dh_out [T,d] (the residual stream's type) is the gradient of h' from the rest
 * of the network (NULL: zero), dn [T,d] bf16 that of n.  h_out is the forward's
 * h' (with b NULL: its h); b, gate, w_post, w_pre as in the forward.
 * With xh = h'/sqrt(mean h'^2 + eps), bh = b/sqrt(mean b^2 + eps), q = dn w_pre:
 *
 *     G      = dh_out + (q - xh mean_i(q xh)) / sqrt(mean h'^2 + eps)
 *     dh     = res_scale G
 *     dgate  = block_scale G u             (summed over the tokens when shared)
 *     p      = block_scale gate G w_post
 *     db     = (p - bh mean_i(p bh)) / sqrt(mean b^2 + eps)       (w_post NULL: p)
 *     dw_pre = sum_t dn xh,   dw_post = sum_t block_scale gate G bh
 *
 * Outputs: dh [T,d] in the residual stream's type (may be dh_out), db [T,d] bf16
 * (may be dn), dgate
 * bf16 [T,d] with ELAS_GATE_TOKEN, else float32 [d]; dw_post, dw_pre float32 [d].
 * Other outputs overlap nothing.  Weight gradients are overwritten, not accumulated,
 * and summed over the tokens in a fixed order in float32.
 * w_pre NULL: dn and h_out are unused and may be NULL, dw_pre is NULL.
 * b NULL: dh is the gradient of h (res_scale unused), db, dgate and dw_post NULL.
 * dh NULL: not written.  Other outputs are required where their operand is given.
 * workspace >= elas_norm_join_bwd_workspace_bytes(T, d, flags) bytes.
 * Sizes as in the forward; T == 0 writes zero weight gradients (only their
 * pointers and the workspace are then inspected).
 */
size_t elas_norm_join_bwd_workspace_bytes(int64_t T, int64_t d, uint32_t flags);
int elas_norm_join_bwd(const void* dh_out, const uint16_t* dn, const void* h_out, const uint16_t* b,
                       const uint16_t* gate, const uint16_t* w_post, const uint16_t* w_pre, int64_t T, int64_t d,
                       float res_scale, float block_scale, float eps, uint32_t flags, void* dh, uint16_t* db,
                       void* dgate, float* dw_post, float* dw_pre, void* workspace, size_t workspace_bytes,
                       void* stream);

/*
 * elas_embed_fwd -- x[t] = scale * table[ids[t]].
 *
 * ids [T] int32 (ELAS_IDS_I64: int64), table [V,d] bf16, x [T,d] bf16
 * (ELAS_RES_F32: float32), rounded once.  An id outside 0 .. V-1 (padding) gives
 * a row of zeros; nothing is read for it.
 * Requires 0 <= T < 2^31, 0 < V < 2^31, d as above, finite scale.  ids need the
 * alignment of their type only.  T == 0 is a no-op.
 */
int elas_embed_fwd(const void* ids, const uint16_t* table, int64_t T, int64_t V, int64_t d, float scale,
                   uint32_t flags, void* x, void* stream);

/*
 * elas_embed_bwd -- dtable[v] = scale * sum of dx[t] over the tokens with
 * ids[t] == v, in float32 and in an order that depends on the ids alone (the
 * tokens are sorted by id first, stably; no floating-point atomics).
 *
 * dx [T,d] bf16 (ELAS_RES_F32: float32); dtable [V,d] float32, every row written
 * (zeros where no token has the id), or with ELAS_EMBED_ADD: the sums are added
 * to it, and rows without tokens are not touched.  Ids outside 0 .. V-1 have no
 * gradient.
 * workspace >= elas_embed_bwd_workspace_bytes(T, V, d, flags) bytes.
 * T == 0 writes zeros (nothing with ELAS_EMBED_ADD).
 */
size_t elas_embed_bwd_workspace_bytes(int64_t T, int64_t V, int64_t d, uint32_t flags);
int elas_embed_bwd(const void* ids, const void* dx, int64_t T, int64_t V, int64_t d, float scale, uint32_t flags,
                   float* dtable, void* workspace, size_t workspace_bytes, void* stream);

/*
 * elas_grad_norm -- norm[0] = sqrt(sum of g^2 over all values of all tensors).
 * elas_grad_clip -- stats[0] = that norm, stats[1] = factor = min(1, max_norm /
 * norm), and every tensor times factor, rounded to its type, in `out`.
 *
 * grads, out   HOST arrays of n device pointers; out[k] has grads[k]'s type and
 *              length and is either grads[k] (in place) or overlaps no tensor.
 *              out NULL: in place.  What is written overlaps no other tensor of
 *              the lists: a tensor given twice would be scaled in a race.
 * numel        HOST array of n lengths >= 0 (a tensor of length 0 may be NULL).
 * dtype        HOST array of n types (ELAS_GRAD_F32 / ELAS_GRAD_BF16).
 * The three arrays are read before the call returns.  Tensors need the alignment
 * of their element only.
 * Squares, sums and the norm are held in 64 bits, so that no norm of finite values
 * overflows before it is rounded to float32; the order of the sum is fixed.  A norm
 * beyond float32's range is reported as infinite and the factor, rounded to float32,
 * with it, but the values are scaled by the factor of the 64-bit norm.
 * Where a value is infinite or NaN the norm is, the factor is 0, and the values are
 * passed on unscaled, so that a program can see what they hold and skip the step.
 * norm / stats: device float32 [1] / [2], 4-byte aligned.
 * Requires 0 <= n < 2^20, fewer than 2^44 values in all, max_norm >= 0 (+inf: never
 * clips).  workspace >= elas_grad_workspace_bytes(n) bytes.
 */
size_t elas_grad_workspace_bytes(int64_t n);
int elas_grad_norm(const void* const* grads, const int64_t* numel, const int32_t* dtype, int64_t n, float* norm,
                   void* workspace, size_t workspace_bytes, void* stream);
int elas_grad_clip(const void* const* grads, void* const* out, const int64_t* numel, const int32_t* dtype, int64_t n,
                   float max_norm, float* stats, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ELAS_TRAIN_H */
