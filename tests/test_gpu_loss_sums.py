"""How exact a row's sum over the vocabulary is where it is long."""
import pytest
import torch

import paper_2605_03667_amd as elas
from oracle import loss as ol

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _roundings(V):
    """Of a sum over V values, by the interface's words: groups of at most 32, of which a thread adds up at most 16 + V /
    8192; then the threads' sums and rescaling, 60 as the oracle counts them."""
    return 32 + 16 + V / 8192 + 60


def _row(x, threads, dtype, large, small):
    """A row whose first pieces of 16 bytes, one to a thread, begin with a value e^19.5 times as likely as the others, so
    that a group of a thread's others is less than half a step of its sum so far."""
    n = 4 if dtype == F32 else 8
    x.fill_(small)
    x[:threads * n:n] = large


def _exact_lse(x, scale):
    return float(torch.logsumexp(x.double() * scale, 0))


@pytest.mark.parametrize("dtype, V", [(F32, 1 << 20), (BF, 1 << 21)])
def test_sum_of_many_small_values(dtype, V):
    """More rows than workgroups of 16 waves are made for, one of which takes part."""
    T = 513
    x = torch.empty((T, V), dtype=dtype, device=DEV)
    _row(x[-1], 256, dtype, 0.0, -18.8 if dtype == F32 else -19.5)
    ids = torch.full((T,), -1, device=DEV)
    ids[-1] = 0
    exact = _exact_lse(x[-1], 1.0)
    # (values below the largest: p |z - max| adds up to 2^-24 20 V / threads at most)
    bound = ol.EPS32 * (_roundings(V) + 4 * 20 * V / 256 * 2.0 ** -24 + 2 + exact)
    lse = elas.elas_token_logp_fwd(x, ids)["lse"][-1]
    assert abs(float(lse) - exact) <= bound, (float(lse) - exact, bound)
    r = elas.elas_token_loss(x, ids, out={"stats": torch.empty(2, device=DEV), "lse": torch.empty(T, device=DEV)})
    assert abs(float(r["lse"][-1]) - exact) <= bound and abs(float(r["stats"][0]) - exact) <= bound
    r = elas.elas_policy_loss(x, ids, torch.ones(T, device=DEV), out={"stats": torch.empty(3, device=DEV), "logp": torch.empty(T, device=DEV)})
    assert abs(float(r["logp"][-1]) + exact) <= bound


def test_sum_anew_of_many_small_values():
    """The gradient at a lse that holds too little: the row's sum is taken anew."""
    V = 1 << 22
    x = torch.empty((1, V), device=DEV)
    _row(x[0], 128, F32, 8192.0, 8192.0 - 18.8)
    lse = torch.full((1,), _exact_lse(x[0], 1.0), device=DEV)
    d = elas.elas_token_logp_bwd(torch.full((1,), -1.0, device=DEV), x, torch.full((1,), V - 1, device=DEV), lse)
    got = d[0, :128 * 4:4].double()
    z = x[0].double()
    want = float(1 / torch.exp(z - z.max()).sum())
    # (the label is elsewhere; 8 roundings for the exponential, the factors and the result)
    rel = ol.EPS32 * (_roundings(V) + 4 * 20 * V / 128 * 2.0 ** -24 + 8)
    assert ((got / want - 1).abs() <= rel).all(), ((got / want - 1).abs().max(), rel)
