"""AdamW in float64 numpy from its definition, with its moments in 32 or 8 bits (oracle;
tests only), and bounds on what float32 arithmetic may differ by.

A code of a first moment holds a sign, 4 bits e and 3 bits f, of a second one e and 4
bits f; with b bits in f it stands for f (e = 0) or (f + 2^b) 2^(e - 1), times its
block's scale.  A magnitude is rounded to one of its two neighbours: up where the 16
random bits of the value reach past the distance to the upper one.
"""
from __future__ import annotations

import numpy as np

from .train import EPS32

BLOCK = 256
TOP = {3: 245760.0, 4: 507904.0}


def values(code, mantissa):
    """What magnitudes' codes stand for, in units of the scale."""
    e, f = code >> mantissa, code & (2 ** mantissa - 1)
    return np.where(e > 0, np.ldexp(f + 2.0 ** mantissa, e - 1), f)


def mix(x):
    x = np.asarray(x, dtype=np.uint64)
    word = np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x6A09E667)) & word
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0xBB67AE85)) & word
    return x ^ (x >> np.uint64(16))


def random_bits(t, tensor, index):
    """32 bits of value ``index`` of tensor ``tensor`` in step t."""
    word = np.uint64(0xFFFFFFFF)
    key = mix(mix((mix(np.uint64(t)) + np.uint64(tensor)) & word))
    return mix((np.asarray(index, dtype=np.uint64) + key) & word)


def codes(y, u, mantissa):
    """Codes of magnitudes y (in units of the scale) with random bits u / 2^16."""
    y = np.asarray(y, dtype=np.float64)
    e = np.maximum(np.frexp(y)[1] - 1 - mantissa, 0)                  # y's neighbours are 2^e apart
    low = np.floor(np.ldexp(y, -e) + u / 65536.0)
    code = np.where(e > 0, (e + 1) * 2.0 ** mantissa + (low - 2.0 ** mantissa), low)
    return np.minimum(code, 2 ** (mantissa + 4) - 1).astype(np.int64)


def blocks(x):
    """x in whole blocks, filled up with zeros."""
    return np.pad(x, (0, -len(x) % BLOCK)).reshape(-1, BLOCK)


def factor(norm, max_norm):
    return 1.0 if norm is None or not norm > max_norm else max_norm / norm


def step(p, g, m, v, t, rate, beta1, beta2, eps, decay, clip=1.0):
    """(p, m, v and their bounds) after step t; the moments are those before rounding to 8 bits."""
    g = g * clip
    m1, v1 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    # the constants, clip and their products: 2 roundings of beta m, 5 of (1 - beta) g, 9 of (1 - beta) g^2; the sum's own
    # and half a step of float32's smallest numbers for what underflows
    tiny = 2.0 ** -148
    m_err = EPS32 * (2 * np.abs(beta1 * m) + 5 * np.abs((1 - beta1) * g) + np.abs(m1)) + tiny
    v_err = EPS32 * (2 * np.abs(beta2 * v) + 9 * (1 - beta2) * g * g + v1) + tiny
    r, root = rate / (1 - beta1 ** t), (1 - beta2 ** t) ** -0.5
    den = np.sqrt(v1) * root + eps
    up = r * m1 / den
    # the denominator: half v's relative error (or the root of all of it, near 0) and 5 roundings (2 of them a root to 1 ulp);
    # a reciprocal to 1 ulp, its product, the rate and its product: 5
    den_err = root * np.where(v1 > 2 * v_err, v_err / np.sqrt(np.maximum(v1, 1e-300)), np.sqrt(v1 + v_err)) + 5 * EPS32 * den
    up_err = r * m_err / den + np.abs(up) * (np.minimum(den_err / np.maximum(den - den_err, eps / 2), 1e3) + 5 * EPS32)
    new = p * (1 - rate * decay) - up
    return new, m1, v1, EPS32 * (3 * np.abs(p) + np.abs(new)) + up_err, m_err, v_err
