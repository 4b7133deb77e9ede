"""elas_token_logp_*, elas_token_loss and elas_policy_loss against the float64 oracle. Tolerances
are the oracle's bounds on float32 arithmetic plus half a step of the output's type."""
import numpy as np
import pytest
import torch

import paper_2605_03667_amd as elas
from oracle import loss as ol

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def _f64(t):
    return t.detach().double().cpu().numpy()


def _near(got, want, bound, dtype=F32, name=""):
    """|got - want| within the bound and half a step of the type, and of its smallest numbers."""
    got = _f64(got)
    half = ol.EPSBF16 if dtype == BF else ol.EPS32
    tiny = 2.0 ** -126          # (numbers under the type's normal range may be taken for 0)
    off = np.abs(got - want) - (bound * (1 + half) + half * np.abs(want) + tiny)
    assert np.all(np.isfinite(got)) and np.all(off <= 0), (name, np.unravel_index(np.argmax(off), off.shape), off.max(), np.abs(got - want).max())


def _inputs(T, V, dtype, seed, pitch=0, shift=0, padding=0.0, banned=0.0, i64=True):
    """Logits about N(0, 4) with the label's raised, in a matrix whose rows begin anywhere; ids, some of
    them outside the vocabulary."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    flat = torch.full((T * (V + pitch) + shift + 8,), 77.0, dtype=dtype, device=DEV)
    x = flat[shift:].as_strided((T, V), (V + pitch, 1), shift)
    x.copy_(torch.randn((T, V), generator=g, device=DEV) * 2)
    if banned:
        x.masked_fill_(torch.rand((T, V), generator=g, device=DEV) < banned, -INF)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV)
    x.scatter_(1, ids[:, None], (torch.randn((T, 1), generator=g, device=DEV) * 3 + np.log(V)).to(dtype))
    if padding:
        u = torch.rand(T, generator=g, device=DEV)
        ids[u < padding] = -1
        ids[u < padding / 2] = V
    return x, ids if i64 else ids.int(), g


def _gradient_like(x, pitch=0, shift=0):
    T, V = x.shape
    flat = torch.full((T * (V + pitch) + shift + 8,), 55.0, dtype=x.dtype, device=DEV)
    return flat, flat[shift:].as_strided((T, V), (V + pitch, 1), shift)


def _check_frame(flat, d):
    """What lies between the gradient's rows is as it was."""
    seen = torch.ones_like(flat, dtype=torch.bool)
    seen.as_strided(d.shape, d.stride(), d.storage_offset()).fill_(False)
    assert (flat[seen] == 55.0).all()


def _check_all(x, ids, g, scale, seed, pitch=0, shift=0):
    """Every call on these logits."""
    T, V = x.shape
    dtype = x.dtype
    n, i = _f64(x), ids.cpu().numpy()
    rand = lambda: torch.randn(T, generator=g, device=DEV)  # noqa: E731
    # log-probabilities
    lp, lse, lp_err, lse_err = ol.logp(n, i, scale)
    out = elas.elas_token_logp_fwd(x, ids, scale=scale)
    _near(out["logp"], lp, lp_err, name="logp")
    _near(out["lse"], lse, lse_err, name="lse")
    # their gradient
    a, b = rand(), rand()
    flat, d = _gradient_like(x, pitch, shift)
    for dlse in (b, None):
        elas.elas_token_logp_bwd(a, x, ids, out["lse"], scale=scale, dlse=dlse, dlogits=d)
        want, err = ol.logp_grad(_f64(a), _f64(b) if dlse is not None else np.zeros(T), n, i, _f64(out["lse"]), scale)
        _near(d, want, err, dtype, "logp_bwd")
    # token loss
    w = (rand().abs() - 0.2).clamp_min(0)
    for weight, z in ((w, 0.01), (None, 0.0)):
        want = ol.token_loss(n, i, None if weight is None else _f64(w), scale, 1 / max(T, 1), z)
        out = elas.elas_token_loss(x, ids, weight=weight, scale=scale, reduce=1 / max(T, 1), z_coef=z,
                                   out={"stats": torch.empty(2, device=DEV), "logp": rand(), "lse": rand(), "dlogits": d})
        for k, t in (("logp", F32), ("lse", F32), ("stats", F32), ("dlogits", dtype)):
            _near(out[k], *want[k], t, k)
    # policy loss
    adv, old = rand(), out["logp"] + 0.3 * rand()
    ref = out["logp"] + torch.where(rand() > 0, 1e-3, 1.0) * rand()
    for o, r, weight, kl in ((old, ref, w, 0.1), (None, ref, None, 0.05), (old, None, None, 0.0), (None, None, w, 0.0), (old, ref, None, 0.0)):
        want, near = ol.policy_loss(n, i, _f64(adv), None if o is None else _f64(o), None if r is None else _f64(r),
                                    None if weight is None else _f64(w), scale, 0.5, 0.2, 0.28, kl)
        assert not near.any()
        out = elas.elas_policy_loss(x, ids, adv, old_logp=o, ref_logp=r, weight=weight, scale=scale, reduce=0.5, clip_low=0.2, clip_high=0.28,
                                    kl_coef=kl, out={"stats": torch.empty(3, device=DEV), "logp": rand(), "dlogits": d})
        for k, t in (("logp", F32), ("stats", F32), ("dlogits", dtype)):
            _near(out[k], *want[k], t, k)
    torch.cuda.synchronize()
    _check_frame(flat, d)


# widths about the pieces of 4 and 8 values, of a wave and of a workgroup
WIDTHS = [1, 2, 3, 7, 8, 9, 63, 255, 256, 257, 511, 513, 1000, 1023, 1025, 2047, 2049, 4096, 5003, 8191, 16385, 32000, 32003, 65537, 131072, 150001]


# widths for the other teams that hold a row (with both types)
TEAMS = [10007, 13001, 15000, 27001, 30001, 48001, 50257, 61003, 64007]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", WIDTHS)
def test_widths(V, dtype):
    T = 37 if V < 5000 else 5
    x, ids, g = _inputs(T, V, dtype, V, padding=0.2)
    _check_all(x, ids, g, 1.25, V)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V, pitch", [(v, p) for v in WIDTHS if v >= 2047 for p in (0, 3)] + [(v, 1) for v in TEAMS])
def test_widths_of_many_tokens(V, pitch, dtype):
    """(Few rows are split over workgroups, many are not.)  300 tokens, 6 of which take part, so that the oracle has few rows
    to compute; all others have results and gradients of 0."""
    T, on = 300, [0, 1, 128, 255, 256, 299]
    x, ids, g = _inputs(T, V, dtype, V, pitch)
    keep = ids.clone()
    ids.fill_(-1)
    ids[on] = keep[on]
    n, i = _f64(x[on]), keep[on].cpu().numpy()
    w = torch.rand(T, generator=g, device=DEV)
    flat, d = _gradient_like(x, pitch)
    out = {"stats": torch.empty(2, device=DEV), "logp": torch.empty(T, device=DEV), "lse": torch.empty(T, device=DEV), "dlogits": d}
    adv = torch.randn(T, generator=g, device=DEV)
    for name, got, want in (("token", elas.elas_token_loss(x, ids, weight=w, scale=1.25, reduce=0.5, z_coef=0.125, out=out),
                             ol.token_loss(n, i, _f64(w[on]), 1.25, 0.5, 0.125)),
                            ("policy", None, ol.policy_loss(n, i, _f64(adv[on]), None, None, _f64(w[on]), 1.25, 0.5, 0.25, 0.25, 0.0)[0])):
        if got is None:
            d.fill_(55.0)
            out = {"stats": torch.empty(3, device=DEV), "logp": torch.empty(T, device=DEV), "dlogits": d}
            got = elas.elas_policy_loss(x, ids, adv, weight=w, scale=1.25, reduce=0.5, clip_low=0.25, clip_high=0.25, out=out)
        for k in want:
            _near(got[k] if k == "stats" else got[k][on], *want[k], dtype if k == "dlogits" else F32, (name, k))
        off = torch.ones(T, dtype=torch.bool, device=DEV)
        off[on] = False
        assert not d[off].any() and not got["logp"][off].any()
        _check_frame(flat, d)
    # in place
    elas.elas_policy_loss(x, ids, adv, weight=w, scale=1.25, reduce=0.5, clip_low=0.25, clip_high=0.25,
                          out={"stats": torch.empty(3, device=DEV), "dlogits": x})
    _near(x[on], *want["dlogits"], dtype, "in place")
    assert not x[off].any()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1, 2, 255, 2048, 2049, 5000])
def test_token_counts(T, dtype):
    x, ids, g = _inputs(T, 301, dtype, T, padding=0.3, i64=False)
    _check_all(x, ids, g, 1.0, T)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V, pitch, shift", [(1000, 24, 0), (1000, 3, 1), (999, 0, 1), (32001, 5, 7), (6, 250, 3), (8192, 1, 0)])
def test_pitches_and_alignments(V, pitch, shift, dtype):
    x, ids, g = _inputs(9, V, dtype, V + pitch, pitch, shift, padding=0.2)
    _check_all(x, ids, g, 0.8, 1, (pitch + 3) % 7, (shift + 1) % 8)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [40, 3000, 40000])
def test_banned_tokens(V, dtype):
    """Logits of -inf, most of a row among them."""
    x, ids, g = _inputs(20, V, dtype, V, banned=0.97)
    x[0, :] = -INF
    x[0, int(ids[0])] = 3.0                       # nothing but the label
    _check_all(x, ids, g, 1.0, 2)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [5, 700, 20000, 140000])
def test_the_types_lowest_value(V, dtype):
    """A row of nothing but a mask's lowest value is a uniform distribution at any scale; beside
    other logits such values have probability 0."""
    low = torch.finfo(dtype).min
    x = torch.full((2, V), low, dtype=dtype, device=DEV)
    x[1, V // 2] = 1.0
    ids = torch.tensor([V - 1, V // 2], device=DEV)
    for scale in (1.0, 3.0, 0.25):
        r = elas.elas_token_loss(x, ids, scale=scale)
        assert abs(float(r["logp"][0]) + np.log(V)) <= 2.0 ** -24 * (V / 64 + 62 + np.log(V))
        want = np.full(V, scale / V)
        want[-1] -= scale
        _near(r["dlogits"][0], want, np.abs(want) * 2.0 ** -24 * (V / 64 + 70), dtype)
        assert float(r["logp"][1]) == 0 and float(r["lse"][1]) == scale
        assert not r["dlogits"][1].any()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [5, 300, 1100, 20001, 70000])
def test_gradient_where_lse_holds_too_little(V, dtype):
    """Logits far from 0, and rows of nothing but the type's lowest value: the gradient of log-probabilities is
    the loss's, and within its bounds (no lse of float32 could give it)."""
    x, ids, g = _inputs(7, V, dtype, V, pitch=3)
    x[1] += 30000.0
    x[2] -= 70000.0
    x[3] = torch.finfo(dtype).min
    x[4] = torch.finfo(dtype).min
    x[4, V // 2] = 0.5
    x[5] += 4000.0
    ids[6] = -1
    w = torch.rand(7, generator=g, device=DEV)
    n, i, wn = _f64(x), ids.cpu().numpy(), _f64(w)
    for scale in (1.0, 0.25, 2.0):
        lse = elas.elas_token_logp_fwd(x, ids, scale=scale)["lse"]
        want = ol.token_loss(n, i, wn, scale, 1.0, 0.0)["dlogits"]
        d = elas.elas_token_logp_bwd(-w, x, ids, lse, scale=scale)
        # rows of a smaller lse: the bound at a given one, and p's change by lse's own error
        lse_err = ol.logp(n, i, scale)[3]
        p = np.exp(scale * (n - n.max(axis=1, keepdims=True)))
        p /= p.sum(axis=1, keepdims=True)
        given = ol.logp_grad(-wn, np.zeros(7), n, i, _f64(lse), scale)[1] + 1.01 * scale * (wn * lse_err)[:, None] * p
        bound = np.where(np.abs(_f64(lse))[:, None] <= 4096, given, want[1])
        _near(d, want[0], bound, dtype, scale)
        y = _gradient_like(x, 3)[1].copy_(x)
        elas.elas_token_logp_bwd(-w, y, ids, lse, scale=scale, dlogits=y)
        _near(y, want[0], bound, dtype, "in place")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [9, 1200, 33000, 132000])
def test_infinities_and_nan_stay_in_their_row(V, dtype):
    x, ids, g = _inputs(6, V, dtype, 3)
    clean = elas.elas_token_loss(x, ids)
    x[1, V // 3] = NAN
    x[2, V // 2] = INF
    x[3, :] = -INF
    x[4, int(ids[4])] = -INF                        # the label itself is banned
    r = elas.elas_token_loss(x, ids)
    assert torch.isnan(r["logp"][1:4]).all() and torch.isnan(r["stats"]).any()
    assert r["lse"][3] == -INF and torch.isnan(r["lse"][1:3]).all()
    assert torch.isnan(r["dlogits"][1:4]).any(1).all()
    assert r["logp"][4] == -INF and torch.isfinite(r["lse"][4]) and torch.isfinite(r["dlogits"][4]).all()
    for k in ("logp", "lse", "dlogits"):
        assert torch.equal(r[k][0], clean[k][0]) and torch.equal(r[k][5], clean[k][5])
    # rows that take no part are not read
    ids[1:5] = -1
    r = elas.elas_token_loss(x, ids, reduce=0.5)
    assert torch.isfinite(r["stats"]).all() and not r["dlogits"][1:5].any() and not r["logp"][1:5].any() and not r["lse"][1:5].any()
    x[0, 0] = NAN
    assert torch.isfinite(elas.elas_token_loss(x, ids, weight=torch.tensor([0.0, 1, 1, 1, 1, 1], device=DEV))["stats"]).all()
    f = elas.elas_token_logp_fwd(x, ids)
    assert torch.isnan(f["logp"][0]) and not f["logp"][1:5].any()
    d = elas.elas_token_logp_bwd(torch.ones(6, device=DEV), x, ids, f["lse"])
    assert torch.isnan(d[0]).all() and not d[1:5].any() and torch.isfinite(d[5]).all()


def _all_near(got, want, dtype):
    for k in got:
        _near(got[k], *want[k], dtype if k == "dlogits" else F32, k)


@pytest.mark.parametrize("gradient", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [100, 5001, 32000])
def test_zeros_beside_exponentials_that_overflow(V, dtype, gradient):
    """kl_coef 0 where the reference is e^200 times as sure of a token (or the policy rules it out), and advantage 0
    where the ratio is e^100: neither takes part."""
    T = 6
    x, ids, g = _inputs(T, V, dtype, V + 5)
    x[0].scatter_(0, ids[:1], -200.0)
    x[1].scatter_(0, ids[1:2], -INF)
    logp = elas.elas_token_logp_fwd(x, ids)["logp"]
    adv, ref = torch.randn(T, generator=g, device=DEV), torch.full((T,), -1.0, device=DEV)
    old = logp.clone()
    old[1] = -2.0          # (its ratio is 0)
    old[2] -= 100.0
    adv[2] = 0.0
    n = _f64(x)
    want, near = ol.policy_loss(np.where(np.isinf(n), -600.0, n), ids.cpu().numpy(), _f64(adv), _f64(old), _f64(ref), None, 1.0, 0.5, 0.2, 0.2, 0.0)
    assert not near.any()
    out = {"stats": torch.empty(3, device=DEV)}
    if gradient:
        out["dlogits"] = torch.empty_like(x)
    elas.elas_policy_loss(x, ids, adv, old_logp=old, ref_logp=ref, reduce=0.5, out=out)
    for k in (0, 2):
        _near(out["stats"][k], want["stats"][0][k], want["stats"][1][k], name=k)
    assert out["stats"][1] == INF
    if gradient:
        _near(out["dlogits"], *want["dlogits"], dtype, "dlogits")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [100, 1000, 5001, 32000, 66000, 140003])
def test_in_place(V, dtype):
    """The gradient over its logits.  A row's values are added up in an order that depends on where its pieces
    of 16 bytes begin, so on its alignment: whatever the order, each of the sum's V values passes through at
    most V / 64 + 60 roundings, which is what the oracle's bounds count.  The gradient at a given lse has no sum: the
    same bits."""
    x, ids, g = _inputs(11, V, dtype, V, pitch=5, padding=0.2)
    n, i = _f64(x), ids.cpu().numpy()
    w = torch.rand(11, generator=g, device=DEV)
    want = elas.elas_token_loss(x, ids, weight=w, z_coef=0.1)
    exact = ol.token_loss(n, i, _f64(w), 1.0, 1.0, float(np.float32(0.1)))
    y = _gradient_like(x, 5)[1]
    y.copy_(x)
    got = elas.elas_token_loss(y, ids, weight=w, z_coef=0.1, out={"stats": torch.empty(2, device=DEV), "dlogits": y})
    _all_near(want, exact, dtype)
    _all_near(got, exact, dtype)
    a = torch.rand(11, generator=g, device=DEV)
    want = elas.elas_token_logp_bwd(a, x, ids, want["lse"])
    y.copy_(x)
    lse = elas.elas_token_logp_fwd(x, ids)["lse"]
    want = elas.elas_token_logp_bwd(a, x, ids, lse)
    elas.elas_token_logp_bwd(a, y, ids, lse, dlogits=y)
    assert torch.equal(y, want)
    y.copy_(x)
    got = elas.elas_policy_loss(y, ids, a, weight=w, out={"stats": torch.empty(3, device=DEV), "dlogits": y})
    exact, _ = ol.policy_loss(n, i, _f64(a), None, None, _f64(w), 1.0, 1.0, 0.2, 0.2, 0.0)
    _all_near(got, exact, dtype)
    # rows that begin alike: the same bits
    y.copy_(x)
    one, two = (elas.elas_token_loss(t, ids, out={"stats": torch.empty(2, device=DEV), "dlogits": t}) for t in (y, _gradient_like(x, 5)[1].copy_(x)))
    assert torch.equal(one["stats"], two["stats"]) and torch.equal(one["dlogits"], two["dlogits"])


@pytest.mark.parametrize("V", [900, 20000])
def test_outputs_that_are_not_wanted(V):
    """A loss without its gradient adds a row's values up in another order: within the same bounds."""
    x, ids, g = _inputs(50, V, BF, 1)
    a = torch.rand(50, generator=g, device=DEV)
    n, i = _f64(x), ids.cpu().numpy()
    alone = elas.elas_token_loss(x, ids, z_coef=0.1, out={"stats": torch.empty(2, device=DEV)})
    _all_near(alone, ol.token_loss(n, i, None, 1.0, 1.0, float(np.float32(0.1))), BF)
    alone = elas.elas_policy_loss(x, ids, a, out={"stats": torch.empty(3, device=DEV)})
    _all_near(alone, ol.policy_loss(n, i, _f64(a), None, None, None, 1.0, 1.0, 0.2, 0.2, 0.0)[0], BF)
    full = elas.elas_token_logp_fwd(x, ids)
    assert torch.equal(elas.elas_token_logp_fwd(x, ids, out={"logp": torch.empty(50, device=DEV)})["logp"], full["logp"])


def test_no_tokens():
    x, ids, a = torch.empty((0, 50), dtype=BF, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV), torch.empty(0, device=DEV)
    for r in (elas.elas_token_loss(x, ids), elas.elas_policy_loss(x, ids, a)):
        assert not r["stats"].any() and r["dlogits"].shape == (0, 50)
    assert elas.elas_token_logp_fwd(x, ids)["logp"].shape == (0,)
    assert elas.elas_token_logp_bwd(a, x, ids, a).shape == (0, 50)
    x, ids, _ = _inputs(300, 50, BF, 1)
    r = elas.elas_token_loss(x, ids - 100)               # none that takes part
    assert not r["stats"].any() and not r["dlogits"].any()


def test_same_bits_every_time():
    x, ids, g = _inputs(3000, 777, BF, 9, padding=0.1)
    first = elas.elas_token_loss(x, ids)
    for _ in range(3):
        again = elas.elas_token_loss(x, ids, workspace=torch.full((elas.elas_token_loss_workspace_bytes(3000, 777),), 255, dtype=torch.uint8, device=DEV))
        assert all(torch.equal(first[k], again[k]) for k in first)


def test_losses_agree_with_the_gradient_of_log_probabilities():
    """A loss's gradient is the gradient of logp and lse applied to its own derivatives (bf16 both,
    half a step each, and float32's errors of two roundings of lse)."""
    x, ids, g = _inputs(64, 2500, F32, 4, padding=0.2)
    f = elas.elas_token_logp_fwd(x, ids, scale=0.9)
    w = torch.rand(64, generator=g, device=DEV)
    r = elas.elas_token_loss(x, ids, weight=w, scale=0.9, reduce=0.5, z_coef=0.02)
    d = elas.elas_token_logp_bwd(-0.5 * w, x, ids, f["lse"], scale=0.9, dlse=0.5 * w * 0.04 * f["lse"])
    assert torch.linalg.norm(r["dlogits"] - d) <= 2e-6 * torch.linalg.norm(d)


def test_gradient_against_differences():
    """Central differences of the loss in a few logits, in float32 logits of a small vocabulary: the
    loss is a sum of 3 terms of about 1, rounded to 2^-24 of itself; at a step of 2^-7 that is 2^-17 a difference, and the
    third derivative's share step^2 / 6 is under 2^-16."""
    x, ids, g = _inputs(3, 6, F32, 8)
    x.clamp_(-2, 2)
    adv, old = torch.tensor([1.0, -1.0, 0.5], device=DEV), torch.tensor([-1.0, -2.0, -1.5], device=DEV)
    calls = [lambda y: elas.elas_token_loss(y, ids, z_coef=0.1, scale=0.9),
             lambda y: elas.elas_policy_loss(y, ids, adv, old_logp=old, ref_logp=old, clip_low=1.0, clip_high=INF, kl_coef=0.1, scale=0.9)]
    for call in calls:
        d = call(x)["dlogits"]
        for t, j in ((0, 0), (1, 3), (2, 5), (0, int(ids[0]))):
            up, down = x.clone(), x.clone()
            up[t, j] += 2.0 ** -7
            down[t, j] -= 2.0 ** -7
            diff = (float(call(up)["stats"][0]) - float(call(down)["stats"][0])) * 64
            assert abs(diff - float(d[t, j])) <= 2.0 ** -14, (t, j, diff, float(d[t, j]))


def test_binding_refusals_on_the_gpu():
    x, ids = torch.zeros((4, 10), dtype=BF, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV)
    a = torch.zeros(4, device=DEV)

    def raises(match, fn, *args, **k):
        with pytest.raises(ValueError, match=match):
            fn(*args, **k)

    for fn in (elas.elas_token_logp_fwd, elas.elas_token_loss):
        raises("ids has shape", fn, x, ids[:3])
        raises("ids must be", fn, x, a)
        raises("ids must be a GPU", fn, x, ids.cpu())
        raises("contiguous rows", fn, x.t(), torch.zeros(10, dtype=torch.int64, device=DEV))
        raises("contiguous", fn, x, torch.zeros((4, 2), dtype=torch.int64, device=DEV)[:, 0])
    raises("weight has shape", elas.elas_token_loss, x, ids, weight=a[:3])
    raises("weight must be", elas.elas_token_loss, x, ids, weight=a.double())
    raises("stats", elas.elas_token_loss, x, ids, out={})
    raises("stats", elas.elas_token_loss, x, ids, out={"stats": a})
    raises("dlogits has shape", elas.elas_token_loss, x, ids, out={"stats": a[:2], "dlogits": x[:3]})
    raises("dlogits must be torch", elas.elas_token_loss, x, ids, out={"stats": a[:2], "dlogits": x.float()})
    raises("overlap", elas.elas_token_loss, x[:, :9], ids, out={"stats": a[:2], "dlogits": x[:, 1:]})
    raises("advantage has shape", elas.elas_policy_loss, x, ids, a[:2])
    raises("old_logp", elas.elas_policy_loss, x, ids, a, old_logp=a[:2])
    raises("lse has shape", elas.elas_token_logp_bwd, a, x, ids, a[:1])
    raises("workspace", elas.elas_token_loss, x, ids, workspace=torch.zeros(64, device=DEV))
    with pytest.raises(elas.ElasError, match="WORKSPACE"):
        elas.elas_token_loss(x, ids, workspace=torch.zeros(8, dtype=torch.uint8, device=DEV))
    with pytest.raises(elas.ElasError, match="ref_logp"):
        elas.elas_policy_loss(x, ids, a, kl_coef=0.1)
    with pytest.raises(elas.ElasError, match="scale"):
        elas.elas_token_loss(x, ids, scale=0.0)
