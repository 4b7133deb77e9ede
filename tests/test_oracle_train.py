"""The float64 oracle of the operators around the FFN, checked on its own: its
gradients against central differences of its forwards, and hand values."""
import numpy as np
import pytest

from oracle import train as ot


def _case(seed, T, d, gate, post, pre, block=True):
    g = np.random.default_rng(seed)
    c = {"h": g.standard_normal((T, d)), "b": None, "gate": None, "w_post": None, "w_pre": None}
    if block:
        c["b"] = g.standard_normal((T, d))
        c["gate"] = {"none": None, "shared": g.standard_normal(d), "token": g.standard_normal((T, d))}[gate]
        c["w_post"] = 1.0 + 0.3 * g.standard_normal(d) if post else None
    c["w_pre"] = 1.0 + 0.3 * g.standard_normal(d) if pre else None
    return c, g.standard_normal((T, d)), g.standard_normal((T, d))


@pytest.mark.parametrize("pre", [False, True])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", ["none", "shared", "token"])
def test_join_gradient_against_differences(gate, post, pre):
    """loss = sum(h' dh + n dn); central differences at step 1e-5 are right to about
    step^2 = 1e-10 and 1e-16 / step = 1e-11, times the loss's curvature (a few tens here)."""
    rs, bs, eps = 0.7, -0.4, 1e-3
    c, dh, dn = _case(3, 3, 8, gate, post, pre)

    def loss(**change):
        h, n = ot.join(**{**c, **change}, res_scale=rs, block_scale=bs, eps=eps)
        return np.sum(h * dh) + (np.sum(n * dn) if pre else 0.0)

    joined, _ = ot.join(**c, res_scale=rs, block_scale=bs, eps=eps)
    got = ot.join_grad(dh, dn if pre else None, joined, c["b"], c["gate"], c["w_post"], c["w_pre"], rs, bs, eps)
    names = {"h": "dh", "b": "db", "gate": "dgate", "w_post": "dw_post", "w_pre": "dw_pre"}
    for name, key in names.items():
        if c[name] is None:
            assert got[key] is None
            continue
        for at in np.ndindex(c[name].shape):
            step = np.zeros_like(c[name])
            step[at] = 1e-5
            diff = (loss(**{name: c[name] + step}) - loss(**{name: c[name] - step})) / 2e-5
            assert abs(diff - got[key][at]) < 1e-7, (key, at)


def test_join_norm_only():
    c, dh, dn = _case(5, 2, 8, "none", False, True, block=False)
    h, n = ot.join(**c, res_scale=9.0, block_scale=9.0, eps=0.0)
    assert np.array_equal(h, c["h"])
    np.testing.assert_allclose(np.mean((n / c["w_pre"]) ** 2, axis=1), 1.0, rtol=1e-12)
    got = ot.join_grad(None, dn, c["h"], None, None, None, c["w_pre"], 9.0, 9.0, 0.0)
    # the norm does not change with the row's length, so its gradient is orthogonal to the row
    assert np.all(np.abs(np.sum(got["dh"] * c["h"], axis=1)) < 1e-12)
    assert got["db"] is None


def test_embedding_and_its_gradient():
    table = np.arange(12.0).reshape(4, 3)
    ids = np.array([2, -1, 0, 2, 4])
    np.testing.assert_array_equal(ot.embed(ids, table, 2.0), 2.0 * np.array([[6, 7, 8], [0, 0, 0], [0, 1, 2], [6, 7, 8], [0, 0, 0]]))
    dx = np.array([[1.0, 2, 3], [9, 9, 9], [4, 5, 6], [10, 20, 30], [9, 9, 9]])
    grad, _, count = ot.embed_grad(ids, dx, 4, 2.0)
    np.testing.assert_array_equal(grad, 2.0 * np.array([[4, 5, 6], [0, 0, 0], [11, 22, 33], [0, 0, 0]]))
    assert list(count) == [1, 0, 2, 0]
    # the lookup is linear in the table: <embed(table), dx> = <table, gradient>
    assert np.sum(ot.embed(ids, table, 2.0) * dx) == np.sum(table * grad)


def test_clip():
    g = [np.array([3.0]), np.array([[0.0, 4.0]])]
    norm, factor, out = ot.clip(g, 1.0)
    assert (norm, factor) == (5.0, 0.2) and np.allclose(out[1], [[0.0, 0.8]])
    assert ot.clip(g, 5.0)[1] == 1.0 and ot.clip([], 1.0)[:2] == (0.0, 1.0)
    assert ot.clip([np.array([np.inf, 1.0])], 1.0)[1] == 0.0
