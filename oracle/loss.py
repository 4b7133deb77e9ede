"""The losses of a training step in float64 numpy from their definitions (oracle; tests
only): log-probabilities of tokens, the token, policy and preference losses, their
gradients, and bounds on what float32 arithmetic may differ by.

With z = scale x, M = max z, a value e = exp(z - M) computed in float32 as
exp2((x - max x) c), c = scale log2(e), has these roundings of 2^-24: the difference, c
(its constant and its product) and the product, each relative to the exponent, so
4 |z - M| in all, and 2 for the exponential.  A value that is rescaled on its way
(its maximum was a smaller one at first) has its exponent in parts that add up to the same
|z - M|, and 3 more roundings a time.  A sum S of V of them in chains of at most V / 64
and a tree on top has at most V / 64 + 60 more, those of the rescaling among them.  So
S has a relative error E of at most 2^-24 (4 sum_j p_j |z_j - M| + V / 64 + 60), and lse
and logp an absolute one of E + 2^-24 (the logarithm of S's mantissa is under 0.35, in float32) before
they are rounded themselves.
"""
from __future__ import annotations

import numpy as np

from .train import EPS32, EPSBF16

__all__ = ["EPS32", "EPSBF16", "keep", "logp", "token_loss", "policy_loss", "preference_loss", "logp_grad"]


def keep(ids, V, weight=None):
    """Tokens that take part."""
    k = (ids >= 0) & (ids < V)
    return k if weight is None else k & (weight != 0)


def _rows(x, ids, scale, on):
    """z - lse, its maximum's distance, and logp, lse of the tokens that take part (0 elsewhere), with E."""
    z = scale * x
    with np.errstate(invalid="ignore", divide="ignore"):
        top = z.max(axis=1, keepdims=True)
        away = np.where(top == z, 0.0, top - z)
        e = np.exp(-away)
        s = e.sum(axis=1, keepdims=True)
        p = e / s
        lse = (top + np.log(s))[:, 0]
        at = np.where(on, ids, 0)
        lp = z[np.arange(len(ids)), at] - top[:, 0] - np.log(s)[:, 0]
        far = np.where(p > 0, away, 0.0)
        E = EPS32 * (4 * (p * far).sum(axis=1) + x.shape[1] / 64 + 60)
    return p, far, np.where(on, lp, 0.0), np.where(on, lse, 0.0), np.where(on, E, 0.0)


def logp(x, ids, scale, weight=None):
    """(logp, lse, bound of logp, bound of lse)."""
    on = keep(ids, x.shape[1], weight)
    _, _, lp, lse, E = _rows(x, ids, scale, on)
    return lp, lse, on * (E + EPS32 * (1 + np.abs(lp))), on * (E + EPS32 * (1 + np.abs(lse)))


def _spread(p, far, ids, on, E, scale, label, label_err, everywhere, every_err):
    """scale (label onehot + everywhere p) and the bound of its error in float32: p's
    relative error is its own exponential's, S's and 4 for the factors."""
    rows = np.arange(len(ids))[on]
    d = scale * everywhere[:, None] * p
    rel = EPS32 * (4 * far + 6) + E[:, None]
    err = scale * ((np.abs(everywhere)[:, None] * rel + every_err[:, None]) * p)
    at = scale * label
    d[rows, ids[on]] += at[on]
    err[rows, ids[on]] += scale * (label_err + 3 * EPS32 * np.abs(label))[on] + EPS32 * np.abs(d[rows, ids[on]])
    d[~on] = err[~on] = 0.0
    return d, err


def logp_grad(dlogp, dlse, x, ids, lse, scale):
    """(dlogits, bound) at a given lse (float32, as the kernel has it): the exponent z - lse has
    roundings of 2^-24 |z| and 3 of |z - lse|, the exponential and the factors 6."""
    on = keep(ids, x.shape[1])
    z = scale * x
    with np.errstate(invalid="ignore", over="ignore"):
        p = np.exp(z - lse[:, None])
        size = np.where(p > 0, np.abs(z) + 3 * np.abs(z - lse[:, None]), 0.0)
    every = dlse - dlogp
    d = scale * every[:, None] * p
    err = np.abs(d) * EPS32 * (size + 6) + scale * EPS32 * (np.abs(dlse) + np.abs(dlogp))[:, None] * p
    rows = np.arange(len(ids))[on]
    d[rows, ids[on]] += scale * dlogp[on]
    err[rows, ids[on]] += EPS32 * (np.abs(scale * dlogp[on]) + np.abs(d[rows, ids[on]]))
    d[~on] = err[~on] = 0.0
    return d, err


def _weights(T, weight, reduce, on):
    return reduce * (np.ones(T) if weight is None else weight) * on


def token_loss(x, ids, weight, scale, reduce, z_coef):
    """dict of (value, bound): logp, lse, stats, dlogits."""
    on = keep(ids, x.shape[1], weight)
    p, far, lp, lse, E = _rows(x, ids, scale, on)
    c = _weights(len(ids), weight, reduce, on)
    z = c * z_coef * lse ** 2
    lse_err = on * (E + EPS32)
    # (c has 2 roundings, the term's factors 3; lse's error counts twice in its square)
    z_err = np.abs(c * z_coef) * (2 * np.abs(lse) * lse_err + 5 * EPS32 * lse ** 2)
    loss = z - c * lp
    loss_err = z_err + np.abs(c) * (lse_err + 2 * EPS32 * np.abs(lp))
    every = c * (1 + 2 * z_coef * lse)
    every_err = np.abs(c) * (2 * abs(z_coef) * (lse_err + 4 * EPS32 * np.abs(lse)) + 4 * EPS32)
    d, d_err = _spread(p, far, ids, on, E, scale, -c, 2 * EPS32 * np.abs(c), every, every_err)
    stats = np.array([loss.sum(), z.sum()])
    stats_err = np.array([loss_err.sum(), z_err.sum()]) + EPS32 * np.abs(stats)
    lp_, lse_, e1, e2 = logp(x, ids, scale, weight)
    return {"logp": (lp_, e1), "lse": (lse_, e2), "stats": (stats, stats_err), "dlogits": (d, d_err)}


def policy_loss(x, ids, advantage, old, ref, weight, scale, reduce, clip_low, clip_high, kl_coef):
    """dict of (value, bound): logp, stats, dlogits; and ``near``: tokens so near a border of the
    clipping that rounding may put them on either side."""
    on = keep(ids, x.shape[1], weight)
    p, far, lp, lse, E = _rows(x, ids, scale, on)
    c = _weights(len(ids), weight, reduce, on)
    lp_err = on * (E + EPS32)
    diff = np.zeros_like(lp) if old is None else on * (lp - old)
    r = np.exp(diff)
    r_rel = np.zeros_like(lp) if old is None else lp_err + EPS32 * (np.abs(diff) + 4)
    lo, hi = 1.0 - clip_low, 1.0 + clip_high
    held = np.where(advantage > 0, r > hi, (advantage < 0) & (r < lo))
    near = on & ((np.abs(r - lo) <= 2 * r * r_rel + 2 * EPS32) | (np.abs(r - hi) <= 2 * r * r_rel + 2 * EPS32))
    bounded = np.clip(r, lo, hi)
    loss = -np.where(held, bounded, r) * advantage
    loss_err = np.abs(advantage) * np.where(held, 3 * EPS32 * bounded, r * (r_rel + 3 * EPS32))
    g = -np.where(held, 0.0, r * advantage)
    g_err = np.where(held, 0.0, np.abs(advantage) * r * (r_rel + 3 * EPS32))
    k, k_err = np.zeros_like(lp), np.zeros_like(lp)
    if ref is not None:
        q = on * (ref - lp)
        q_err = lp_err + EPS32 * np.abs(q)
        k = np.expm1(q) - q
        # (its derivative is exp(q) - 1; the series or expm1 and the difference: 12 roundings of the terms' sizes)
        k_err = np.abs(np.expm1(q)) * q_err + 12 * EPS32 * np.where(np.abs(q) < 0.5, k, np.abs(np.expm1(q)) + np.abs(q)) + q_err ** 2
        loss = loss + kl_coef * k
        loss_err = loss_err + abs(kl_coef) * k_err + 2 * EPS32 * np.abs(kl_coef * k)
        g = g - kl_coef * np.expm1(q)
        g_err = g_err + abs(kl_coef) * (np.exp(q) * q_err + 4 * EPS32 * np.abs(np.expm1(q)))
    g_err = g_err + 2 * EPS32 * np.abs(g)
    terms = np.stack([c * loss, c * k, c * held])
    errs = np.stack([np.abs(c) * (loss_err + 4 * EPS32 * np.abs(loss)), np.abs(c) * (k_err + 3 * EPS32 * k), 3 * EPS32 * np.abs(c * held)])
    label, label_err = c * g, np.abs(c) * (g_err + 3 * EPS32 * np.abs(g))
    d, d_err = _spread(p, far, ids, on, E, scale, label, label_err, -label, label_err)
    stats = terms.sum(axis=1)
    return {"logp": logp(x, ids, scale, weight)[::2], "stats": (stats, errs.sum(axis=1) + EPS32 * np.abs(stats)), "dlogits": (d, d_err)}, near


def preference_loss(logp, ref, offsets, beta, smoothing):
    """dict(stats, margin, dlogp); sums are 64-bit, so each is the float32 nearest to it or next to that."""
    diff = logp if ref is None else logp - ref
    pairs = len(offsets) // 2
    margin, dlogp, loss = np.zeros(pairs), np.zeros(len(logp)), 0.0
    for i in range(pairs):
        a, b, c = offsets[2 * i:2 * i + 3]
        z = margin[i] = beta * (diff[a:b].sum() - diff[b:c].sum())
        soft = np.log1p(np.exp(-abs(z)))
        loss += (1 - smoothing) * (soft + max(-z, 0.0)) + smoothing * (soft + max(z, 0.0))
        g = (smoothing * np.exp(-max(-z, 0.0) - soft) - (1 - smoothing) * np.exp(-max(z, 0.0) - soft)) * beta / pairs
        dlogp[a:b] = g
        dlogp[b:c] = -g
    n = max(pairs, 1)
    return {"stats": np.array([loss / n, (margin > 0).sum() / n, margin.sum() / n]), "margin": margin, "dlogp": dlogp}
