"""The operators around the FFN in a training step, in float64 numpy from their
definitions (oracle; tests only): the norms before and after a block with its
gate and residual scale, the embedding and the clipping of gradients, their
gradients, and bounds on what float32 arithmetic may differ by.

The pre-norm residual architecture is Sec. 4.1's: norms are root-mean-square
norms, v / sqrt(mean(v^2) + eps) over the features, times a gain.
"""
from __future__ import annotations

import numpy as np

EPS32 = 2.0 ** -24        # half an ulp of float32 (24 significant bits), relative
EPSBF16 = 2.0 ** -8       # half an ulp of bf16 (8 significant bits), relative
TINY_BF16 = 2.0 ** -133   # spacing of bf16's subnormals


def rms(v, eps):
    return 1.0 / np.sqrt(np.mean(v * v, axis=-1, keepdims=True) + eps)


def join(h, b, gate, w_post, w_pre, res_scale, block_scale, eps):
    """(h', n) of the norm join; absent operands are None."""
    if b is not None:
        u = b if w_post is None else b * rms(b, eps) * w_post
        h = res_scale * h + block_scale * (1.0 if gate is None else gate) * u
    return h, None if w_pre is None else h * rms(h, eps) * w_pre


def join_grad(dh, dn, h, b, gate, w_post, w_pre, res_scale, block_scale, eps):
    """Gradients at the joined stream h, as dict(dh, db, dgate, dw_post, dw_pre);
    absent operands give None."""
    out = dict.fromkeys(("dh", "db", "dgate", "dw_post", "dw_pre"))
    shape = (h if dh is None else dh).shape
    G = np.zeros(shape) if dh is None else dh
    if w_pre is not None:
        s = rms(h, eps)
        q = dn * w_pre
        G = G + s * q - h * s ** 3 * np.mean(q * h, axis=-1, keepdims=True)
        out["dw_pre"] = np.sum(dn * h * s, axis=0)
    out["dh"] = G if b is None else res_scale * G
    if b is None:
        return out
    r = 1.0 if w_post is None else rms(b, eps)
    u = b * r * (1.0 if w_post is None else w_post)
    if gate is not None:
        dg = block_scale * G * u
        out["dgate"] = dg if gate.ndim == 2 else dg.sum(axis=0)
    p = block_scale * G * (1.0 if gate is None else gate)
    if w_post is None:
        out["db"] = p
    else:
        out["dw_post"] = np.sum(p * b * r, axis=0)
        p = p * w_post
        out["db"] = r * p - b * r ** 3 * np.mean(p * b, axis=-1, keepdims=True)
    return out


def _steps(d):
    """Roundings on the way of one value through a row's sum (a chain over a lane's
    share of the row, at most d / 64 values, then a tree) and the operations around it."""
    return d / 64 + 40


def join_error(h, b, gate, w_post, w_pre, res_scale, block_scale, eps):
    """Bounds on |computed - exact| of (h', n) in float32 arithmetic before the
    final rounding: every value is a sum of terms of the sizes below, each with at
    most _steps(d) roundings of 2^-24, and n inherits h's error directly and through
    its norm."""
    d = h.shape[-1]
    k = _steps(d) * EPS32
    size = np.abs(h)
    if b is not None:
        u = b if w_post is None else b * rms(b, eps) * w_post
        size = abs(res_scale) * size + np.abs(block_scale * (1.0 if gate is None else gate) * u)
    he = k * size if b is not None else 0.0 * size
    if w_pre is None:
        return he, None
    hj, _ = join(h, b, gate, w_post, w_pre, res_scale, block_scale, eps)
    s = rms(hj, eps)
    ms = np.mean(hj * hj, axis=-1, keepdims=True) + eps
    norm_rel = np.mean(np.abs(hj) * he, axis=-1, keepdims=True) / ms
    return he, np.abs(w_pre) * s * (he + np.abs(hj) * (k + norm_rel))


def join_grad_error(dh, dn, h, b, gate, w_post, w_pre, res_scale, block_scale, eps, tokens):
    """The same for the gradients: the sizes of all terms, added up without signs,
    times the roundings on their way (two sums over the row, and for the sums over
    the tokens one addition per token)."""
    d = (h if dh is None else dh).shape[-1]
    k = 2 * _steps(d) * EPS32
    a = lambda v: None if v is None else np.abs(v)  # noqa: E731
    s = None if w_pre is None else rms(h, eps)
    size = np.zeros((h if dh is None else dh).shape) if dh is None else np.abs(dh)
    out = dict.fromkeys(("dh", "db", "dgate", "dw_post", "dw_pre"))
    kt = k + tokens * EPS32
    if w_pre is not None:
        q = a(dn) * a(w_pre)
        size = size + s * q + a(h) * s ** 3 * np.mean(q * a(h), axis=-1, keepdims=True)
        out["dw_pre"] = kt * np.sum(a(dn) * a(h) * s, axis=0)
    out["dh"] = k * size * (1.0 if b is None else abs(res_scale))
    if b is None:
        return out
    r = 1.0 if w_post is None else rms(b, eps)
    p = abs(block_scale) * size
    if gate is not None:
        dg = p * a(b) * r * (1.0 if w_post is None else a(w_post))
        out["dgate"] = k * dg if gate.ndim == 2 else kt * dg.sum(axis=0)
        p = p * a(gate)
    if w_post is None:
        out["db"] = k * p
    else:
        out["dw_post"] = kt * np.sum(p * a(b) * r, axis=0)
        p = p * a(w_post)
        out["db"] = k * (r * p + a(b) * r ** 3 * np.mean(p * a(b), axis=-1, keepdims=True))
    return out


def embed(ids, table, scale):
    inside = (ids >= 0) & (ids < table.shape[0])
    return np.where(inside[..., None], scale * table[np.where(inside, ids, 0)], 0.0)


def embed_grad(ids, dx, V, scale):
    """(dtable, its float32 error bound, tokens per row)."""
    out, size, count = np.zeros((V, dx.shape[-1])), np.zeros((V, dx.shape[-1])), np.zeros(V, dtype=np.int64)
    for i, row in zip(ids.reshape(-1), dx.reshape(-1, dx.shape[-1])):
        if 0 <= i < V:
            out[i] += row
            size[i] += np.abs(row)
            count[i] += 1
    return scale * out, (count[:, None] + 3) * EPS32 * abs(scale) * size, count


def clip(grads, max_norm):
    """(norm, factor, clipped): nothing is scaled where the norm is not finite."""
    norm = float(np.sqrt(sum(np.sum(np.square(g.astype(np.float64))) for g in grads)))
    if not np.isfinite(norm):
        return norm, 0.0, list(grads)
    factor = max_norm / norm if norm > max_norm else 1.0
    return norm, factor, [factor * g for g in grads]
