/*
 * elas_adamw.h -- C ABI of the update of a training step: AdamW over many
 * tensors at once, with its moments in 32 or 8 bits, the clipping by the gradients'
 * norm folded in, and bf16 copies of the weights written in the same pass.  Part of libelas;
 * the conventions, status codes, debug mode and timing calls of elas.h hold here too.
 */
#ifndef ELAS_ADAMW_H
#define ELAS_ADAMW_H

#include "elas_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Values that share a scale of moments in 8 bits; every tensor's moments begin a block. */
#define ELAS_ADAMW_BLOCK    256
/* elas_adam8_values: the codes are second moments. */
#define ELAS_ADAM8_SECOND   2u

/*
 * elas_adamw_step -- one step over n tensors:
 *
 *     t = step + 1,  g' = g min(1, max_norm / norm)                       (norm NULL: g)
 *     m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2
 *     p = (1 - lr decay_k) p - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 *
 * with lr = rate, times rate_factor[0] where that is given.  p's update uses m and v before they are
 * rounded to 8 bits; the arithmetic is float32, with factors of the step found in 64 bits.
 *
 * params, grads  HOST arrays of n device pointers; types as in elas_grad_clip
 *                (ELAS_GRAD_F32 / ELAS_GRAD_BF16), a type for each tensor in
 *                param_dtype and grad_dtype.  A bf16 p is rounded to nearest.
 * copies         HOST array of n device pointers, or NULL; copies[k] (or NULL) receives p
 *                as bf16, rounded to nearest.
 * numel, decay   HOST arrays of n lengths (>= 0) and weight decays (finite).
 * The arrays are read before the call returns.  Tensors need their element's alignment
 * only.  What is written (params, copies, moments, step) overlaps nothing else of the call: ELAS_ERR_OVERLAP
 * between the moments, step, norm, rate_factor, workspace and anything; tensors of the lists are
 * not compared with one another.
 * Tensor k's moments begin at value 256 sum_{j<k} ceil(numel[j] / 256) of m and v; what fills
 * up its last block is written as 0.  There are `blocks` = sum_k ceil(numel[k] / 256).
 * bits 32: m, v float32 [256 blocks]; m_scale, v_scale NULL.
 * bits 8:  m, v uint8 [256 blocks], m_scale, v_scale float32 [blocks].  A code stands for a
 *          multiple of its block's scale: with f its lowest 3 bits (m; 4 for v) and e the 4 bits
 *          above, f where e = 0, else (f + 8) 2^(e-1) (v: f + 16); m's highest bit is its
 *          sign.  The scale is the block's largest magnitude / 245760 (v: 507904), rounded up
 *          where that is below 2^-126.  A magnitude
 *          is rounded to one of its two neighbours by chance, so that its expectation is
 *          its value and averages that move by less than a step move all the same; the
 *          random bits are a hash of t, k and the value's index (32 bits of it), so a step can be repeated.
 *          A v above 0 is never rounded to 0.  A block that a value which is not finite gets
 *          into has a scale that is not finite either.
 * step           device int64 [1], 8-byte aligned: steps taken; raised by 1 in the call.
 * norm           device float32 [1] (as elas_grad_norm gives it) or NULL.  Where it is
 *                infinite or NaN the step is skipped: nothing changes, step neither.
 * rate_factor    device float32 [1] or NULL: a schedule that a captured graph can follow.
 * m, v and the scales are 16-byte aligned.
 * Requires 0 <= n < 2^20, fewer than 2^40 values in all, 0 <= beta < 1, finite rate and
 * eps >= 2^-126 (all in float32), max_norm >= 0, step >= 0.  workspace >= elas_adamw_workspace_bytes() bytes.
 */
size_t elas_adamw_workspace_bytes(void);
int elas_adamw_step(void* const* params, const void* const* grads, uint16_t* const* copies, const int64_t* numel,
                    const int32_t* param_dtype, const int32_t* grad_dtype, const float* decay, int64_t n, int bits, void* m,
                    float* m_scale, void* v, float* v_scale, int64_t* step, double rate, const float* rate_factor,
                    double beta1, double beta2, double eps, const float* norm, double max_norm, void* workspace,
                    size_t workspace_bytes, void* stream);

/*
 * elas_adam8_values -- what 8-bit codes of first moments (ELAS_ADAM8_SECOND: second ones) stand
 * for: out [256 blocks] bf16, or float32 with ELAS_RES_F32.  codes, scale and out 16-byte
 * aligned.  Requires 0 <= blocks < 2^32.
 */
int elas_adam8_values(const uint8_t* codes, const float* scale, int64_t blocks, uint32_t flags, void* out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ELAS_ADAMW_H */
