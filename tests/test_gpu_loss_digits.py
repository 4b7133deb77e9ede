"""The gradient of log-probabilities where a float32 lse holds too little of a row's sum."""
import numpy as np
import pytest
import torch

import paper_2605_03667_amd as elas
from oracle import loss as ol

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("V", [5, 300, 1100, 20001, 70000])
def test_float32_gradient_keeps_its_digits(V):
    """float32 logits at some distance from 0: the gradient at their lse is within the bounds of the loss's own, which has
    the row's sum and not a rounded logarithm of it; up to 64 within those at a given lse and of that lse's rounding."""
    shifts = [0.0, 30.0, 100.0, -100.0, 333.0, -700.0, 1500.0, -2500.0, 3000.0, 3800.0, 4000.0, -4000.0]
    T = len(shifts)
    g = torch.Generator(device=DEV)
    g.manual_seed(V)
    x = torch.randn((T, V), generator=g, device=DEV) * 2 + torch.tensor(shifts, device=DEV)[:, None]
    ids = torch.randint(0, V, (T,), generator=g, device=DEV)
    w = 0.1 + torch.rand(T, generator=g, device=DEV)
    n, i, wn = x.double().cpu().numpy(), ids.cpu().numpy(), w.double().cpu().numpy()
    lse = elas.elas_token_logp_fwd(x, ids)["lse"]
    d = elas.elas_token_logp_bwd(-w, x, ids, lse).double().cpu().numpy()
    want, own = ol.token_loss(n, i, wn, 1.0, 1.0, 0.0)["dlogits"]
    l64 = lse.double().cpu().numpy()
    p = np.exp(n - n.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    given = ol.logp_grad(-wn, np.zeros(T), n, i, l64, 1.0)[1] + 1.01 * (wn * ol.logp(n, i, 1.0)[3])[:, None] * p
    bound = np.where(np.abs(l64)[:, None] <= 64, given, own)
    off = np.abs(d - want) - (bound * (1 + ol.EPS32) + ol.EPS32 * np.abs(want) + 2.0 ** -126)
    assert np.all(off <= 0), (V, [float(s) for s, o in zip(shifts, off.max(axis=1)) if o > 0])
