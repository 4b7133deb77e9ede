"""The losses and log-probabilities on the kernels that a call reaches by its sizes and by the outputs that it wants: without a
gradient and with many rows, and teams that take several rows in turn.  Against the float64 oracle, with its bounds."""
import numpy as np
import pytest
import torch

import paper_2605_03667_amd as elas
from oracle import loss as ol

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _f64(t):
    return t.detach().double().cpu().numpy()


def _near(got, want, bound, dtype, name):
    got = _f64(got)
    half = ol.EPSBF16 if dtype == BF else ol.EPS32
    off = np.abs(got - want) - (bound * (1 + half) + half * np.abs(want) + 2.0 ** -126)
    assert np.all(np.isfinite(got)) and np.all(off <= 0), (name, np.unravel_index(np.argmax(off), off.shape), off.max())


def _rows(T, V, on, dtype, seed, pitch=3):
    """Logits and ids of T tokens, those of ``on`` taking part; the others' logits are NaN, so that a result that read
    them shows it."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.full((T, V + pitch), float("nan"), dtype=dtype, device=DEV)[:, :V]
    some = (torch.randn((len(on), V), generator=g, device=DEV) * 2).to(dtype)
    label = torch.randint(0, V, (len(on),), generator=g, device=DEV)
    some.scatter_(1, label[:, None], (torch.randn((len(on), 1), generator=g, device=DEV) * 3 + np.log(V)).to(dtype))
    at = torch.tensor(on, device=DEV)
    x[at] = some
    ids = torch.full((T,), -1, device=DEV)
    ids[at] = label
    return x, ids, at, _f64(some), label.cpu().numpy(), g


def _check(x, ids, at, n, i, g, dtype, gradient):
    """Token and policy loss and the log-probabilities, with or without gradients."""
    T = len(ids)
    off = torch.ones(T, dtype=torch.bool, device=DEV)
    off[at] = False
    new = lambda *s: torch.full(s, 7.0, device=DEV)  # noqa: E731
    w, adv = 0.1 + torch.rand(T, generator=g, device=DEV), torch.randn(T, generator=g, device=DEV)

    def results(got, want):
        for k in got:
            _near(got[k] if k == "stats" else got[k][at], *want[k], dtype if k == "dlogits" else F32, k)
            if k != "stats":
                assert not got[k][off].any(), k

    def out(**more):
        return {**more, **({"dlogits": torch.full_like(x, 7.0)} if gradient else {})}

    results(elas.elas_token_loss(x, ids, weight=w, scale=1.25, reduce=0.5, z_coef=0.125, out=out(stats=new(2), logp=new(T), lse=new(T))),
            ol.token_loss(n, i, _f64(w[at]), 1.25, 0.5, 0.125))
    logp, lse, logp_err, lse_err = ol.logp(n, i, 1.25)
    old = new(T)
    # (no ratio so near a border of the clipping that rounding decides on which side it is)
    change = 0.3 * torch.randn(len(at), generator=g, device=DEV)
    for border in (-np.log(0.75), -np.log(1.25)):
        change = torch.where((change - border).abs() < 1e-3, change + 3e-3, change)
    old[at] = torch.tensor(logp, device=DEV).float() + change
    ref = old + 0.1
    want, near = ol.policy_loss(n, i, _f64(adv[at]), _f64(old[at]), _f64(ref[at]), _f64(w[at]), 1.25, 0.5, 0.25, 0.25, 0.125)
    assert not near.any()
    results(elas.elas_policy_loss(x, ids, adv, old_logp=old, ref_logp=ref, weight=w, scale=1.25, reduce=0.5, clip_low=0.25, clip_high=0.25,
                                  kl_coef=0.125, out=out(stats=new(3), logp=new(T))), want)
    results(elas.elas_token_logp_fwd(x, ids, scale=1.25, out={"logp": new(T), "lse": new(T)}), {"logp": (logp, logp_err), "lse": (lse, lse_err)})


@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [900, 9001, 20000, 66001])
@pytest.mark.parametrize("T", [97, 129, 300, 512, 513, 700])
def test_many_rows(T, V, dtype, gradient):
    on = sorted({0, 1, T // 3, T // 2, T - 2, T - 1})
    x, ids, at, n, i, g = _rows(T, V, on, dtype, T + V)
    _check(x, ids, at, n, i, g, dtype, gradient)


@pytest.mark.parametrize("V, dtype, gradient", [(7000, BF, True), (9000, BF, False), (500, BF, True), (5001, F32, False), (20000, BF, True),
                                                (13001, F32, True), (66000, BF, True)])
def test_teams_that_take_rows_in_turn(V, dtype, gradient):
    """More rows than workgroups (8192, of 4 rows each where a wave takes a row): row t and row t + 8192 (32768) come one
    after the other in one team, with a barrier a row, and both take part."""
    wide = V * (2 if dtype == BF else 4) > 100000
    turn = 32768 if V <= 600 else 8192
    first = range(0, 300, 30 if wide else 3)
    on = sorted([*first, *(t + turn for t in first)])
    x, ids, at, n, i, g = _rows(turn + 300, V, on, dtype, V)
    _check(x, ids, at, n, i, g, dtype, gradient)
