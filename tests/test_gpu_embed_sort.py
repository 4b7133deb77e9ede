"""The sorts of the embedding's gradient at every number of tokens to a thread and to a
workgroup, and of passes.  The gradients are small whole numbers, whose sums are exact
in float32 in any order, so that a token in the wrong row or counted twice shows."""
import pytest
import torch

import paper_2605_03667_amd as elas

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _memory():
    yield
    torch.cuda.empty_cache()


def _check(T, V, kind, add, res=BF, d=8):
    g = torch.Generator(device=DEV)
    g.manual_seed(T + V)
    u = torch.rand(T, generator=g, device=DEV, dtype=torch.float64)
    if kind == "words":        # about the inverse of the rank
        ids = (torch.exp(u * torch.log(torch.tensor(V + 1.0, dtype=torch.float64))) - 1).long().clamp_(max=V - 1)
    elif kind == "high":       # keys that differ in their last digit
        ids = V - 1 - (u * 5).long() * ((V - 1) // 5)
    else:
        ids = (u * V).long().clamp_(max=V - 1)
    ids[torch.rand(T, generator=g, device=DEV) < 0.05] = -1
    ids[-1], ids[0] = V - 1, 0
    ids = ids.to(torch.int32)
    dx = torch.randint(-4, 5, (T, d), generator=g, device=DEV, dtype=torch.int8).to(res)
    before = torch.randint(-9, 10, (V, d), generator=g, device=DEV, dtype=torch.int8).float() if add else torch.zeros((V, d), device=DEV)
    inside = ids >= 0
    want = before.clone().index_add_(0, ids[inside], 2 * dx[inside].float())
    table = before if add else torch.full((V, d), float("nan"), device=DEV)
    got = elas.elas_embed_bwd(ids, dx, V, 2.0, dtable=table, accumulate=add)
    assert got is table and torch.equal(got, want)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("kind", ["words", "uniform"])
@pytest.mark.parametrize("T", [512 * 8192, 512 * 8192 + 1, 3 * 512 * 8192 + 77])
def test_several_tiles_to_a_workgroup(T, kind, add):
    """Above 4 M tokens a workgroup takes more than one tile of 8192: two passes."""
    _check(T, 32000, kind, add)


@pytest.mark.parametrize("V", [300, 2 ** 20])
def test_several_tiles_one_and_three_passes(V):
    _check(512 * 8192 * 2 + 4099, V, "words", False)


def test_order_of_several_tiles():
    """A row's tokens stay in their order: the same tokens, sorted beforehand, give the same
    bits, which sums of about 130 values of a row in another order hardly do."""
    T, V, d = 512 * 8192 + 9000, 32000, 8
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    dx = torch.randn((T, d), generator=g, device=DEV)
    got = elas.elas_embed_bwd(ids, dx, V)
    order = torch.argsort(ids, stable=True)
    assert torch.equal(elas.elas_embed_bwd(ids[order].contiguous(), dx[order].contiguous(), V), got)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("kind", ["words", "uniform", "high"])
@pytest.mark.parametrize("T", [131072, 131073, 262144, 262145, 1000003])
def test_tokens_to_a_thread(T, kind, add):
    """1 token of a tile to a thread up to 131072, 4 up to 262144, then 8."""
    _check(T, 32000, kind, add, F32 if T % 2 else BF)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("kind", ["words", "uniform", "high"])
@pytest.mark.parametrize("V", [2 ** 18, 2 ** 27])
@pytest.mark.parametrize("T", [8193, 20000, 140000])
def test_three_and_four_passes(T, V, kind, add):
    _check(T, V, kind, add)


def test_one_pass():
    for T in (8193, 131073, 300000):
        for V in (1, 2, 511):
            _check(T, V, "uniform", False)
