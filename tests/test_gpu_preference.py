"""elas_preference_loss against the float64 oracle.  Sums and the loss are 64-bit: results are the
float32 nearest to the oracle's, or one beside it where the sum's order (2^-53 of its terms) decides."""
import numpy as np
import pytest
import torch

import paper_2605_03667_amd as elas
from oracle import loss as ol

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _case(lengths, seed, before=0, behind=0, ref=True, i64=True, sigma=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    offsets = np.concatenate([[0], np.cumsum(lengths)]) + before
    n = int(offsets[-1]) + behind
    logp = -torch.rand(n, generator=g, device=DEV) * sigma
    r = logp + 0.3 * sigma * torch.randn(n, generator=g, device=DEV) if ref else None
    return logp, r, torch.tensor(offsets, dtype=torch.int64 if i64 else torch.int32, device=DEV)


def _verify(logp, ref, offsets, beta, smoothing):
    host = [None if t is None else t.double().cpu().numpy() for t in (logp, ref)]
    want = ol.preference_loss(*host, offsets.cpu().numpy(), float(np.float32(beta)), float(np.float32(smoothing)))
    got = elas.elas_preference_loss(logp, offsets, ref, beta, smoothing)
    size = float(np.abs(host[0]).sum() + (0 if ref is None else np.abs(host[1]).sum()))
    noise = len(host[0]) * 2.0 ** -53 * size * abs(beta)
    for k, w in want.items():
        g = got[k].double().cpu().numpy()
        # (a number below float32's normal range: a step of 2^-149)
        # dlogp's relative change with z is at most 1 a unit of z, and its two sigmoids, each to 2e-10 of itself, may cancel
        rel = 2.0 ** -24 * 1.01 + (noise if k == "dlogp" else 0.0)
        both = 2e-10 * abs(beta) / max(len(offsets) // 2, 1) * min(smoothing, 1 - smoothing) if k == "dlogp" else 0.0
        assert np.all(np.abs(g - w) <= rel * np.abs(w) + both + 2.0 ** -149 + (0.0 if k == "dlogp" else noise)), (k, np.abs(g - w).max())
    alone = elas.elas_preference_loss(logp, offsets, ref, beta, smoothing, out={"stats": torch.empty(3, device=DEV)})
    assert torch.equal(alone["stats"], got["stats"])
    inplace = logp.clone()
    elas.elas_preference_loss(inplace, offsets, ref, beta, smoothing, out={"stats": torch.empty(3, device=DEV), "dlogp": inplace})
    assert torch.equal(inplace, got["dlogp"])


@pytest.mark.parametrize("smoothing", [0.0, 0.1, 1.0])
@pytest.mark.parametrize("lengths", [[1, 1], [0, 3], [3, 0], [0, 0], [255, 256], [257, 1, 64, 63], [5000, 1023, 1, 0, 0, 7, 1025, 2]])
def test_lengths(lengths, smoothing):
    for before, behind in ((0, 0), (3, 700)):
        for ref in (True, False):
            _verify(*_case(lengths, sum(lengths), before, behind, ref, i64=ref), 0.1, smoothing)


@pytest.mark.parametrize("pairs", [1, 100, 2048, 2049, 5000])
def test_many_pairs(pairs):
    lengths = np.random.default_rng(pairs).integers(0, 40, 2 * pairs)
    _verify(*_case(lengths, pairs, 1, 1, i64=False), 0.5, 0.1)


def test_a_long_answer():
    _verify(*_case([300000, 123457], 1), 0.01, 0.0)


def test_large_margins():
    """No overflow either way."""
    for sign in (1.0, -1.0):
        logp = torch.tensor([-1e6 * (sign < 0), -1e6 * (sign > 0), 0.0, 0.0], device=DEV)
        offsets = torch.tensor([0, 1, 2, 3, 4], device=DEV)
        _verify(logp, None, offsets, 1.0, 0.0)
        _verify(logp, None, offsets, 1.0, 0.25)
    for value in (float("inf"), float("-inf"), float("nan")):
        x = torch.tensor([value, -1.0, -2.0, -3.0], device=DEV)
        r = elas.elas_preference_loss(x, torch.tensor([0, 1, 2, 3, 4], device=DEV))
        z = 0.1 * (value + 1.0)
        assert np.array_equal(r["margin"].cpu().numpy()[:1], np.float32([z]), equal_nan=True) and float(r["margin"][1]) == pytest.approx(0.1)
        g = r["dlogp"].cpu().numpy()
        assert np.isnan(g[:2]).all() if value != value else g[0] == (0.0 if value > 0 else -np.float32(0.1) / 2)
        assert np.isfinite(g[2:]).all()


@pytest.mark.parametrize("smoothing", [0.0, 0.25, 1.0])
def test_gradients_of_far_margins(smoothing):
    """A sigmoid near 0 is not 1 less one near 1: the gradient keeps its relative precision at both ends."""
    for z in (-60.0, -33.0, -20.0, 20.0, 33.0, 60.0):
        logp = torch.tensor([z, 0.0], device=DEV)
        _verify(logp, None, torch.tensor([0, 1, 2], device=DEV), 1.0, smoothing)


def test_no_pairs():
    r = elas.elas_preference_loss(torch.ones(500, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV))
    assert not r["stats"].any() and not r["dlogp"].any() and r["margin"].shape == (0,)
    r = elas.elas_preference_loss(torch.ones(0, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV))
    assert r["stats"].tolist() == [pytest.approx(np.log(2), rel=2.0 ** -23), 0.0, 0.0]


def test_offsets_out_of_range_are_held_to_the_tensor():
    """Each to 0 .. N: such a call reads and writes nothing outside."""
    flat = torch.full((300,), -1.0, device=DEV)
    inside = flat[100:200]
    out = torch.full((300,), 5.0, device=DEV)
    for off in ([-50, 20, 1000], [0, 2 ** 31 - 1, 2 ** 31 - 1], [90, 50, 10], [-2 ** 31, -5, 40]):
        r = elas.elas_preference_loss(inside, torch.tensor(off, dtype=torch.int32, device=DEV), beta=1.0,
                                      out={"stats": torch.empty(3, device=DEV), "margin": torch.empty(1, device=DEV), "dlogp": out[100:200]})
        a, b, c = np.clip(off, 0, 100)
        assert float(r["margin"]) == -max(b - a, 0) + max(c - b, 0)
        assert (out[:100] == 5).all() and (out[200:] == 5).all()


def test_gradient_against_differences():
    """The margin is linear in logp, so a change of 1/4 in one value moves the loss by the integral of its
    gradient: half the two gradients' sum, up to beta^3 / (12 64) of curvature and roundings of the loss, 2^-24 each."""
    logp, ref, offsets = _case([3, 2, 4, 1], 5)
    base = elas.elas_preference_loss(logp, offsets, ref, 0.5, 0.1)
    for j in range(10):
        moved = logp.clone()
        moved[j] += 0.25
        other = elas.elas_preference_loss(moved, offsets, ref, 0.5, 0.1)
        diff = (float(other["stats"][0]) - float(base["stats"][0])) / 0.25
        assert abs(diff - 0.5 * (float(base["dlogp"][j]) + float(other["dlogp"][j]))) <= 0.125 / 768 + 2.0 ** -21


def test_refusals_on_the_gpu():
    x, y, off = torch.zeros(10, device=DEV), torch.zeros(10, device=DEV), torch.tensor([0, 5, 10], device=DEV)

    def raises(match, *a, **k):
        with pytest.raises(ValueError, match=match):
            elas.elas_preference_loss(*a, **k)

    raises("ref_logp has shape", x, off, x[:5])
    raises("logp must be torch.float32", x.double(), off)
    raises("offsets must be a GPU", x, off.cpu())
    raises("margin", x, off, out={"stats": x[:3], "margin": x[:2]})
    raises("stats", x, off, out={"margin": x[:1]})
    raises("overlap", x[:8], off.clamp_max(8), out={"stats": x[:3].clone(), "dlogp": x[1:9]})
    raises("overlap", x, off, y, out={"stats": x[:3].clone(), "dlogp": y})
    raises("contiguous", torch.zeros((10, 2), device=DEV)[:, 0], off)
    with pytest.raises(elas.ElasError, match="smoothing"):
        elas.elas_preference_loss(x, off, smoothing=1.5)
