"""Element offsets past 2^32: rows, answers and values at the far end of tensors of more than four
billion values come out as they do alone."""
import numpy as np
import pytest
import torch

import paper_2605_03667_amd as elas
from oracle import adamw as oa

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _memory():
    yield
    torch.cuda.empty_cache()


def test_logits():
    T, V = 135_000, 32_000          # 4.3e9
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = torch.zeros((T, V), dtype=BF, device=DEV)
    ids = torch.full((T,), -1, device=DEV)
    rows = torch.randn((5, V), generator=g, device=DEV).to(BF)
    x[-5:] = rows
    ids[-5:] = torch.randint(0, V, (5,), generator=g, device=DEV)
    want = elas.elas_token_loss(rows, ids[-5:], z_coef=0.1)
    dlogits = torch.ones_like(x)
    got = elas.elas_token_loss(x, ids, z_coef=0.1, out={"stats": torch.empty(2, device=DEV), "logp": torch.empty(T, device=DEV),
                                                        "lse": torch.empty(T, device=DEV), "dlogits": dlogits})
    for k in ("logp", "lse", "dlogits"):
        assert torch.equal(got[k][-5:], want[k]), k
    assert torch.allclose(got["stats"], want["stats"], rtol=2.0 ** -23)
    assert not got["logp"][:-5].any() and not dlogits[:3].any() and not dlogits[-8:-5].any()
    f = elas.elas_token_logp_fwd(x, ids)
    assert torch.equal(f["logp"][-5:], elas.elas_token_logp_fwd(rows, ids[-5:])["logp"])
    a = torch.rand(T, generator=g, device=DEV)
    dlogits.fill_(1.0)
    elas.elas_token_logp_bwd(a, x, ids, f["lse"], dlogits=dlogits)
    assert torch.equal(dlogits[-5:], elas.elas_token_logp_bwd(a[-5:].clone(), rows, ids[-5:], f["lse"][-5:].clone()))
    assert not dlogits[-8:-5].any() and not dlogits[:3].any()


def test_a_pitch_past_four_billion_values():
    """Few rows far apart."""
    V, pitch = 500, 1_500_000_000
    flat = torch.zeros(3 * pitch + V, dtype=BF, device=DEV)
    x = flat.as_strided((4, V), (pitch, 1))
    rows = torch.randn((4, V), device=DEV).to(BF)
    x.copy_(rows)
    ids = torch.tensor([1, 2, 3, 4], device=DEV)
    want = elas.elas_token_loss(rows, ids)
    got = elas.elas_token_loss(x, ids, out={"stats": torch.empty(2, device=DEV), "logp": torch.empty(4, device=DEV), "dlogits": x})
    assert torch.allclose(got["logp"], want["logp"], rtol=2.0 ** -20) and torch.allclose(x.float(), want["dlogits"].float(), rtol=2.0 ** -7)


def test_preference():
    N = (1 << 32) + 1000
    logp = torch.zeros(N, device=DEV)
    logp[-700:] = -torch.rand(700, device=DEV)
    offsets = torch.tensor([N - 700, N - 400, N - 100], device=DEV)
    want = elas.elas_preference_loss(logp[-700:].clone(), torch.tensor([0, 300, 600], device=DEV))
    dlogp = torch.ones(N, device=DEV)
    got = elas.elas_preference_loss(logp, offsets, out={"stats": torch.empty(3, device=DEV), "margin": torch.empty(1, device=DEV), "dlogp": dlogp})
    # (the sums' orders differ: 2^-53 of 300 terms each, before the rounding to float32)
    assert torch.allclose(got["margin"], want["margin"], rtol=2.0 ** -23) and torch.allclose(got["stats"], want["stats"], rtol=2.0 ** -23)
    assert torch.allclose(dlogp[-700:], want["dlogp"], rtol=2.0 ** -23) and not dlogp[-100:].any()
    assert not dlogp[: 1 << 20].any() and not dlogp[N - (1 << 20):N - 700].any()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(bits):
    """Two tensors, so that the second's moments lie past 2^32 values too."""
    n, tail = (1 << 32) + 300, 600
    p = [torch.zeros(n, dtype=BF, device=DEV), torch.ones(tail, device=DEV)]
    g = [torch.zeros(n, dtype=BF, device=DEV), torch.randn(tail, device=DEV)]
    g[0][-tail:] = torch.randn(tail, device=DEV).to(BF)
    p[0][-tail:] = 0.5
    opt = elas.ElasAdamW(p, bits=bits, decay=0.1)
    want = []
    for k in range(2):
        x = p[k][-tail:].double().cpu().numpy()
        want.append(oa.step(x, g[k][-tail:].double().cpu().numpy(), 0 * x, 0 * x, 1, 0.01, 0.9, 0.999, 1e-8, 0.1))
    elas.elas_adamw_step(opt, g, 0.01)
    last = -(-n // 256)
    for k, half in ((0, 2.0 ** -8), (1, 2.0 ** -24)):
        got = p[k][-tail:].double().cpu().numpy()
        assert np.all(np.abs(got - want[k][0]) <= want[k][3] * 1.01 + half * np.abs(want[k][0]))
        at = (n - tail) if k == 0 else last * 256
        if bits == 32:
            assert np.all(np.abs(opt.m[at:at + tail].double().cpu().numpy() - want[k][1]) <= want[k][4] + 2.0 ** -24 * np.abs(want[k][1]))
        else:
            m = elas.elas_adam8_values(opt.m, opt.m_scale, dtype=BF)[at:at + tail].double().cpu().numpy()
            # a neighbour: an eighth of the value away at most, and half a step of bf16
            assert np.all(np.abs(m - want[k][1]) <= (1 / 8 + 2.0 ** -8) * np.abs(want[k][1]) + np.abs(want[k][1]).max() / oa.TOP[3])
    assert not p[0][: 1 << 20].any() and not p[0][n - (1 << 20):n - tail].any()


def test_adamw_of_more_pieces_than_a_grid_has_threads_for():
    """2^34 values in pieces of 1024, a workgroup of 256 threads to each, would be 2^32 threads."""
    n, tail = (1 << 34) + 300, 600
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, dtype=BF, device=DEV)
    ends = (slice(0, tail), slice(n - tail, n))
    for at in ends:
        p[at], g[at] = 0.5, torch.randn(tail, device=DEV).to(BF)
    want = []
    for at in ends:
        x = p[at].double().cpu().numpy()
        want.append(oa.step(x, g[at].double().cpu().numpy(), 0 * x, 0 * x, 1, 0.01, 0.9, 0.999, 1e-8, 0.0))
    opt = elas.ElasAdamW([p], bits=8)
    elas.elas_adamw_step(opt, [g], 0.01)
    assert int(opt.step) == 1
    for at, w in zip(ends, want):
        assert np.all(np.abs(p[at].double().cpu().numpy() - w[0]) <= w[3] * 1.01 + 2.0 ** -24 * np.abs(w[0]))
    assert not p[tail: 1 << 20].any() and not p[n - (1 << 20):n - tail].any()


def test_values_of_more_codes_than_a_grid_has_threads_for():
    """2^35 codes, 8 to a thread."""
    blocks = (1 << 27) + 3
    codes, scale = torch.zeros(256 * blocks, dtype=torch.uint8, device=DEV), torch.ones(blocks, device=DEV)
    some = torch.randint(0, 256, (700,), dtype=torch.uint8, device=DEV)
    codes[:700], codes[-700:] = some, some
    want = elas.elas_adam8_values(torch.cat([some, some.new_zeros(68)]), scale[:3].clone())[:700]
    got = elas.elas_adam8_values(codes, scale)
    assert torch.equal(got[:700], want) and torch.equal(got[-700:], want)
    assert not got[700: 1 << 20].any() and not got[256 * blocks - (1 << 20):-700].any()
