"""The float64 oracles of the losses and of AdamW, checked on their own: gradients against
central differences, the 8-bit format and its rounding, hand values."""
import numpy as np
import pytest

from oracle import adamw as oa
from oracle import loss as ol


def _differences(f, x, at, step=1e-5):
    d = np.zeros_like(x)
    d[at] = step
    return (f(x + d) - f(x - d)) / (2 * step)


def _inputs(seed, T=5, V=7):
    g = np.random.default_rng(seed)
    ids = np.array([3, 0, -1, V, V - 1])[:T]
    return g, g.standard_normal((T, V)), ids


@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_token_loss_gradient(scale):
    """Central differences at step 1e-5 are right to 1e-10 times third derivatives of a few and 1e-16 / 1e-5."""
    g, x, ids = _inputs(1)
    w = np.array([0.5, 2.0, 1.0, 1.0, 0.0])
    loss = lambda y: ol.token_loss(y, ids, w, scale, 0.3, 0.05)["stats"][0][0]  # noqa: E731
    got = ol.token_loss(x, ids, w, scale, 0.3, 0.05)["dlogits"][0]
    for at in np.ndindex(x.shape):
        assert abs(_differences(loss, x, at) - got[at]) < 1e-9
    assert not got[2:].any()


@pytest.mark.parametrize("seed", [0, 1, 2])
@pytest.mark.parametrize("with_old, with_ref", [(True, True), (True, False), (False, True)])
def test_policy_loss_gradient(with_old, with_ref, seed):
    """(No token's ratio lies within 1e-3 of a border.)  Without old log-probabilities the ratio is
    exp(logp - logp') with logp' held fixed."""
    g, x, ids = _inputs(seed + 10)
    adv = g.standard_normal(5)
    lp = ol.logp(x, ids, 1.3)[0]
    old = lp + np.array([0.5, -0.6, 0.0, 0.0, 0.05])
    ref = lp + g.standard_normal(5) if with_ref else None

    def call(y, o):
        return ol.policy_loss(y, ids, adv, o, ref, None, 1.3, 0.25, 0.2, 0.3, 0.1)[0]

    got = call(x, old if with_old else None)["dlogits"][0]
    for at in np.ndindex(x.shape):
        assert abs(_differences(lambda y: call(y, old if with_old else lp)["stats"][0][0], x, at) - got[at]) < 1e-8
    if not with_old:
        assert call(x, None)["stats"][0][0] == pytest.approx(call(x, lp)["stats"][0][0], rel=1e-12)


def test_logp_gradient():
    g, x, ids = _inputs(3)
    a, b = g.standard_normal(5), g.standard_normal(5)
    on = ol.keep(ids, 7)

    def loss(y):
        lp, lse, _, _ = ol.logp(y, ids, 0.8)
        return (a * lp + b * lse)[on].sum()

    got = ol.logp_grad(a, b, x, ids, ol.logp(x, ids, 0.8)[1], 0.8)[0]
    for at in np.ndindex(x.shape):
        assert abs(_differences(loss, x, at) - got[at]) < 1e-9


def test_preference_gradient():
    g = np.random.default_rng(5)
    offsets = np.array([1, 4, 4, 9, 10, 12, 15])
    logp, ref = g.standard_normal(17), g.standard_normal(17)
    call = lambda y: ol.preference_loss(y, ref, offsets, 0.7, 0.2)  # noqa: E731
    got = call(logp)
    for at in range(17):
        assert abs(_differences(lambda y: call(y)["stats"][0], logp, at) - got["dlogp"][at]) < 1e-9
    assert not got["dlogp"][[0, 15, 16]].any()
    for z in (800.0, -800.0):        # no overflow
        r = ol.preference_loss(np.array([z]), None, np.array([0, 1, 1]), 1.0, 0.0)
        assert r["stats"][0] == pytest.approx(max(-z, 0.0), abs=1e-300) and r["dlogp"][0] == pytest.approx(-1.0 if z < 0 else 0.0, abs=1e-300)


def test_logp_of_masked_rows():
    x = np.array([[-np.inf, 2.0, -np.inf], [-3e38, -3e38, -3e38], [0.0, 1.0, 2.0]])
    lp, lse, _, _ = ol.logp(x, np.array([1, 0, 7]), 1.0)
    assert lp[0] == 0 and lse[0] == 2 and abs(lp[1] + np.log(3)) < 1e-12 and lp[2] == 0 and lse[2] == 0


@pytest.mark.parametrize("mantissa", [3, 4])
def test_codes(mantissa):
    """Codes rise with their values; a value that a code stands for keeps it whatever the random bits;
    one between two codes becomes the upper one for the distance's share of the random bits."""
    every = np.arange(2 ** (mantissa + 4))
    v = oa.values(every, mantissa)
    assert np.all(np.diff(v) > 0) and v[-1] == oa.TOP[mantissa] and v[0] == 0 and v[1] == 1
    for u in (0, 1, 65535):
        assert np.array_equal(oa.codes(v, u, mantissa), every)
    for c in (0, 1, 2 ** mantissa - 1, 2 ** mantissa, 3 * 2 ** mantissa + 1, 2 ** (mantissa + 4) - 2):
        for share in (0.25, 0.5, 0.8125):
            y = v[c] + share * (v[c + 1] - v[c])
            got = oa.codes(np.full(65536, y), np.arange(65536), mantissa)
            assert set(got) == {c, c + 1} and (got == c + 1).sum() == share * 65536


def test_mix_is_a_bijection_and_bits_are_even():
    """Distinct inputs give distinct words; each bit is set in half of 2^17 words, within 6 deviations of sqrt(2^17) / 2."""
    w = oa.random_bits(7, 3, np.arange(1 << 17))
    assert len(np.unique(w)) == 1 << 17
    for b in range(32):
        assert abs(int(((w >> np.uint64(b)) & np.uint64(1)).sum()) - (1 << 16)) < 6 * (1 << 17) ** 0.5 / 2


def test_step_by_hand():
    p, m, v, *_ = oa.step(np.array([1.0]), np.array([2.0]), np.array([0.0]), np.array([0.0]), 1, 0.1, 0.9, 0.99, 1e-9, 0.5)
    # the first step's moments, unbiased, are g and g^2: a step of the rate, and of rate * decay
    assert m[0] == pytest.approx(0.2) and v[0] == pytest.approx(0.04) and p[0] == pytest.approx(1 - 0.05 - 0.1)
    p, m, v, *_ = oa.step(np.array([1.0]), np.array([2.0]), np.array([0.0]), np.array([0.0]), 1, 0.1, 0.9, 0.99, 1e-9, 0.5, clip=oa.factor(4.0, 1.0))
    assert m[0] == pytest.approx(0.05) and oa.factor(0.5, 1.0) == 1.0 and oa.factor(None, 0.0) == 1.0
