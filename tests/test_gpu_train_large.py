"""Element offsets past 2^32: rows at the far end of tensors of more than four
billion values come out as they do alone, bit for bit."""
import pytest
import torch

import paper_2605_03667_amd as elas

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
T, D = 2_100_000, 2048          # 4.3e9 values


@pytest.fixture(autouse=True)
def _memory():
    yield
    torch.cuda.empty_cache()


def _ends(t):
    return torch.cat([t[:3], t[-5:]])


def test_norm_join():
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    rows = [torch.randn((8, D), generator=g, device=DEV).to(BF) for _ in range(3)]
    gate, w1, w2 = (torch.randn(D, generator=g, device=DEV).to(BF) for _ in range(3))
    big = [torch.zeros((T, D), dtype=BF, device=DEV) for _ in range(3)]
    for t, r in zip(big, rows):
        t[:3], t[-5:] = r[:3], r[3:]
    h, b, dn = big
    want = elas.elas_norm_join_fwd(rows[0], rows[1], gate, w1, w2, block_scale=0.5)
    got = elas.elas_norm_join_fwd(h, b, gate, w1, w2, block_scale=0.5)
    assert torch.equal(_ends(got["h"]), want["h"]) and torch.equal(_ends(got["n"]), want["n"])
    want_g = elas.elas_norm_join_bwd(None, rows[2], want["h"], rows[1], gate, w1, w2, block_scale=0.5)
    got_g = elas.elas_norm_join_bwd(None, dn, got["h"], b, gate, w1, w2, block_scale=0.5)
    assert torch.equal(_ends(got_g["dh"]), want_g["dh"]) and torch.equal(_ends(got_g["db"]), want_g["db"])
    # all other rows are zero and add nothing; the order of the few terms may differ
    for k in ("dgate", "dw_post", "dw_pre"):
        assert torch.allclose(got_g[k], want_g[k], rtol=0, atol=16 * 2.0 ** -24 * float(want_g[k].abs().max() * 8))


def test_embedding():
    table = torch.zeros((T, D), dtype=BF, device=DEV)
    table[-2:] = torch.randn((2, D), device=DEV).to(BF)
    ids = torch.tensor([T - 1, 0, T - 2, T, T - 1], device=DEV)
    x = elas.elas_embed_fwd(ids, table)
    assert torch.equal(x[0], table[-1]) and torch.equal(x[2], table[-2]) and not x[1].any() and not x[3].any()
    assert torch.equal(x[4], x[0])
    del table
    grad = torch.full((T, D), float("nan"), device=DEV)
    elas.elas_embed_bwd(ids, x, T, dtable=grad)
    assert torch.equal(grad[-1], 2 * x[0].float()) and torch.equal(grad[-2], x[2].float())
    assert not grad[:-2].any()


def test_long_token_list():
    """dx of more than 2^32 values."""
    n, d = T, D
    dx = torch.zeros((n, d), dtype=BF, device=DEV)
    dx[-1], dx[0] = 1.0, 2.0
    ids = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    ids[-1], ids[0], ids[n // 2] = 7, 7, 3
    grad = elas.elas_embed_bwd(ids, dx, 10)
    assert (grad[7] == 3.0).all() and not grad[[0, 1, 2, 3, 4, 5, 6, 8, 9]].any()


def test_clip():
    g = torch.zeros(T * D + 3, dtype=BF, device=DEV)
    g[-1], g[0], g[2 ** 32 + 1] = 3.0, 4.0, 12.0
    stats = elas.elas_grad_clip([g], 6.5)
    assert stats.tolist() == [13.0, 0.5]
    assert float(g[-1]) == 1.5 and float(g[0]) == 2.0 and float(g[2 ** 32 + 1]) == 6.0 and int(torch.count_nonzero(g)) == 3
