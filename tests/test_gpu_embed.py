"""elas_embed_fwd / _bwd against the float64 oracle: the lookup is one float32
product and one rounding, so it must agree bit for bit; a row of the gradient is
a float32 sum, which must lie within one rounding per token of its terms' sizes."""
import numpy as np
import pytest
import torch

import paper_2605_03667_amd as elas
from oracle import bf16 as obf
from oracle import train as ot

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _ids(kind, T, V, seed):
    g = np.random.default_rng(seed)
    if kind == "uniform":
        ids = g.integers(0, V, T)
    elif kind == "words":       # about the inverse of the rank
        ids = np.minimum((np.exp(g.random(T) * np.log(V + 1.0)) - 1.0).astype(np.int64), V - 1)
    elif kind == "one":         # every token the same
        ids = np.full(T, V // 2)
    elif kind == "last":
        ids = np.full(T, V - 1)
    elif kind == "padding":
        ids = np.full(T, -1)
    elif kind == "ends":        # the table's ends, and ids just outside it
        ids = g.choice([0, V - 1, V, -1, -2], T)
    else:                       # half padding, the rest few rows with long runs
        ids = np.where(g.random(T) < 0.5, -1, g.integers(0, min(V, 3), T))
    return ids


def _dx(T, d, dtype, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn((T, d), generator=g, device=DEV).to(dtype)


@pytest.mark.parametrize("res", [BF, F32])
@pytest.mark.parametrize("i64", [False, True])
@pytest.mark.parametrize("T,V,d", [(1, 1, 8), (1, 32000, 2048), (5, 7, 520), (333, 1000, 768), (64, 300, 4104), (7, 20, 65536)])
def test_lookup_bits(T, V, d, i64, res):
    ids = _ids("ends" if T == 333 else "uniform", T, V, T)
    table = _dx(V, d, BF, V)
    scale = 1.7
    dev_ids = torch.from_numpy(ids).to(DEV, torch.int64 if i64 else torch.int32)
    x = elas.elas_embed_fwd(dev_ids, table, scale, dtype=res)
    torch.cuda.synchronize()
    t64 = table.float().cpu().numpy()
    inside = (ids >= 0) & (ids < V)
    want = np.where(inside[:, None], np.float32(scale) * t64[np.where(inside, ids, 0)], np.float32(0))
    if res == BF:
        assert np.array_equal(obf.from_f64(x.double().cpu().numpy()), obf.from_f64(want.astype(np.float64)))
    else:
        assert np.array_equal(x.cpu().numpy(), want)


def test_lookup_shapes_and_wide_ids():
    """Ids of any shape; 64-bit ids are compared as such (2^32 + 3 is no row 3)."""
    table = _dx(10, 16, BF, 1)
    ids = torch.tensor([[3, 2 ** 32 + 3], [-2 ** 40, 9]], device=DEV)
    x = elas.elas_embed_fwd(ids, table)
    assert x.shape == (2, 2, 16)
    assert torch.equal(x[0, 0], table[3]) and torch.equal(x[1, 1], table[9])
    assert not x[0, 1].any() and not x[1, 0].any()
    grad = elas.elas_embed_bwd(ids, x, 10)
    assert torch.equal(grad[3], table[3].float()) and torch.equal(grad[9], table[9].float())
    assert not grad[[0, 1, 2, 4, 5, 6, 7, 8]].any()


def _check_grad(ids, dx, V, scale, got, before=None):
    ref, bound, count = ot.embed_grad(ids, dx.double().cpu().numpy(), V, scale)
    g = got.double().cpu().numpy()
    if before is not None:
        b = before.double().cpu().numpy()
        ref, bound = ref + b, bound + (2 + count[:, None]) * ot.EPS32 * np.abs(b)
        assert np.array_equal(g[count == 0], b[count == 0])      # not touched
    else:
        assert not g[count == 0].any()
    bound = bound + ot.EPS32 * np.abs(ref) + 2.0 ** -149
    bad = ~(np.abs(g - ref) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(), g[bad][:3], ref[bad][:3])


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("kind", ["uniform", "words", "one", "last", "padding", "ends", "runs"])
@pytest.mark.parametrize("T,V,d", [(1, 1, 8), (65, 64, 24), (3000, 257, 136), (20000, 1000, 40)])
def test_gradient(T, V, d, kind, add):
    ids = _ids(kind, T, V, T + V)
    dx = _dx(T, d, BF, T)
    before = _dx(V, d, F32, 3)
    table = before.clone() if add else torch.full((V, d), float("nan"), device=DEV)
    got = elas.elas_embed_bwd(torch.from_numpy(ids).to(DEV), dx, V, 0.5, dtable=table, accumulate=add)
    assert got is table
    _check_grad(ids, dx, V, 0.5, got, before if add else None)


@pytest.mark.parametrize("T,V,d,res,i64", [(2048, 32000, 512, BF, True), (511, 32000, 768, F32, False), (4096, 70000, 264, BF, False),
                                           (300, 2 ** 21 + 5, 8, F32, True), (600, 2 ** 23 + 1, 8, BF, False), (300, 50, 2048, BF, True), (100, 40, 2056, F32, False),
                                           (40, 9, 65536, BF, True), (16384, 32000, 64, BF, False), (16385, 32000, 64, BF, False),
                                           (70001, 5000, 32, BF, True)])
def test_gradient_sizes(T, V, d, res, i64):
    ids = _ids("words", T, V, 5)
    dx = _dx(T, d, res, 6)
    dev_ids = torch.from_numpy(ids).to(DEV, torch.int64 if i64 else torch.int32)
    got = elas.elas_embed_bwd(dev_ids, dx, V, 3.0)
    _check_grad(ids, dx, V, 3.0, got)


def test_same_bits_every_time_and_in_any_workspace():
    T, V, d = 30011, 3000, 256
    ids = torch.from_numpy(_ids("words", T, V, 8)).to(DEV, torch.int32)
    dx = _dx(T, d, BF, 9)
    ref = elas.elas_embed_bwd(ids, dx, V, 1.5)
    need = elas.elas_embed_bwd_workspace_bytes(T, V, d, 0)
    for fill in (0x00, 0xFF, 0x7F):
        ws = torch.full((need,), fill, dtype=torch.uint8, device=DEV)
        assert torch.equal(elas.elas_embed_bwd(ids, dx, V, 1.5, workspace=ws), ref)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("T", [33, 64, 1024, 1025, 2049, 4096, 4097])
def test_long_rows_among_short_ones(T, add):
    """Rows of one, 32, 33 and many tokens side by side, cut between waves and workgroups."""
    g = np.random.default_rng(T)
    V, d = 600, 520
    sizes = g.choice([1, 2, 31, 32, 33, 64, 65, 500], 400)
    ids = np.repeat(g.permutation(V)[:400], sizes)[:T]
    ids = np.concatenate([ids, np.full(T - len(ids), V - 1)])
    ids = g.permutation(ids)
    dx = _dx(T, d, BF, T)
    before = _dx(V, d, F32, 3)
    table = before.clone() if add else torch.full((V, d), float("nan"), device=DEV)
    got = elas.elas_embed_bwd(torch.from_numpy(ids).to(DEV), dx, V, 0.5, dtable=table, accumulate=add)
    _check_grad(ids, dx, V, 0.5, got, before if add else None)
    again = before.clone() if add else torch.empty_like(table)
    assert torch.equal(elas.elas_embed_bwd(torch.from_numpy(ids).to(DEV), dx, V, 0.5, dtable=again, accumulate=add), got)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("T", [511, 512, 513, 4096])
@pytest.mark.parametrize("kind", ["folded", "distance"])
def test_ids_that_meet_in_one_workgroup(T, add, kind):
    """Few tokens: the rows are dealt out to 256 workgroups (added) or 512 (written) by their
    ids' bits folded together; ids whose fold is the same, and ids at equal distances."""
    V, d = 2 ** 20 + 3, 8
    bits = 8 if add else 9
    g = np.random.default_rng(T)
    q = g.integers(0, (V >> bits) - 1, T)
    ids = q << bits | ((q ^ q >> bits ^ 5) & ((1 << bits) - 1)) if kind == "folded" else q << bits
    dx = _dx(T, d, BF, T)
    before = _dx(V, d, F32, 3)
    table = before.clone() if add else torch.full((V, d), float("nan"), device=DEV)
    got = elas.elas_embed_bwd(torch.from_numpy(ids).to(DEV), dx, V, 0.5, dtable=table, accumulate=add)
    _check_grad(ids, dx, V, 0.5, got, before if add else None)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("kind", ["uniform", "words", "one", "padding", "ends", "runs"])
@pytest.mark.parametrize("T", [4097, 5151, 8191, 8192, 8193])
def test_between_one_launch_and_the_radix_sort(T, kind, add):
    V, d = 2500, 40
    ids = _ids(kind, T, V, T)
    dx = _dx(T, d, F32, T)
    before = _dx(V, d, F32, 3)
    table = before.clone() if add else torch.full((V, d), float("nan"), device=DEV)
    got = elas.elas_embed_bwd(torch.from_numpy(ids).to(DEV), dx, V, 0.5, dtable=table, accumulate=add)
    _check_grad(ids, dx, V, 0.5, got, before if add else None)


def test_nonfinite_gradients_stay_in_their_row():
    T, V, d = 5000, 300, 128
    ids_np = _ids("words", T, V, 4)
    ids = torch.from_numpy(ids_np).to(DEV)
    dx = _dx(T, d, BF, 2)
    ref = elas.elas_embed_bwd(ids, dx, V)
    dx[17, 3] = float("inf")
    got = elas.elas_embed_bwd(ids, dx, V)
    rows = torch.ones(V, dtype=torch.bool, device=DEV)
    rows[ids_np[17]] = False
    assert torch.equal(got[rows], ref[rows]) and torch.isinf(got[ids_np[17], 3])


def test_no_tokens():
    ids = torch.empty(0, dtype=torch.int32, device=DEV)
    dx = torch.empty((0, 16), dtype=BF, device=DEV)
    assert elas.elas_embed_fwd(ids, _dx(4, 16, BF, 1)).shape == (0, 16)
    assert not elas.elas_embed_bwd(ids, dx, 4).any()
    table = _dx(4, 16, F32, 2)
    keep = table.clone()
    assert torch.equal(elas.elas_embed_bwd(ids, dx, 4, dtable=table, accumulate=True), keep)
