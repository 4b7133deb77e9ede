"""The entry points of include/elas_loss.h and include/elas_adamw.h on the host: exported,
and refusing every invalid argument with its status before anything is launched (so
these calls never touch a GPU); the binding's checks of shapes, types, strides and devices."""
import ctypes
import os
import re

import pytest
import torch

import paper_2605_03667_amd as elas
from paper_2605_03667_amd import loss as binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.skipif(not os.path.exists(elas.LIB_PATH), reason="libelas.so not built")

A = 0x10000            # aligned, never dereferenced: every call below fails validation
NULL, SHAPE, ALIGN, WORKSPACE, FLAGS = 1, 2, 3, 4, 5
BF, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("header, functions, constants", [("elas_loss.h", 7, 1), ("elas_adamw.h", 3, 2)])
def test_exports_and_constants(header, functions, constants):
    text = open(os.path.join(ROOT, "include", header)).read()
    names = set(re.findall(r"\b(elas_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert len(names) == functions and names <= set(elas._SIGNATURES)
    handle = ctypes.CDLL(elas.LIB_PATH)
    assert all(hasattr(handle, n) for n in names)
    defines = dict(re.findall(r"#define\s+(ELAS_[A-Z0-9_]+)\s+([0-9]+)u?", text))
    assert len(defines) == constants
    for k, v in defines.items():
        assert getattr(elas, k) == int(v), k
    assert names <= set(elas.__all__)


def _status(name, defaults, **kw):
    assert set(kw) <= set(defaults)
    return getattr(elas.lib(), name)(*{**defaults, **kw}.values(), None)


WS = dict(ws=A, wsb=1 << 20)
LOGITS = dict(x=A, ld=16, ids=A, T=4, V=10, scale=1.0, flags=0)


def _fwd(**kw):
    return _status("elas_token_logp_fwd", {**LOGITS, "logp": A, "lse": A}, **kw)


def _bwd(**kw):
    return _status("elas_token_logp_bwd", dict(dlogp=A, dlse=A, x=A, ld=16, ids=A, lse=A, T=4, V=10, scale=1.0, flags=0, d=2 * A, ldo=16), **kw)


def _loss(**kw):
    return _status("elas_token_loss", dict(x=A, ld=16, ids=A, w=A, T=4, V=10, scale=1.0, reduce=1.0, z=0.0, flags=0, logp=A, lse=A, d=2 * A, ldo=16,
                                           stats=A, **WS), **kw)


def _policy(**kw):
    return _status("elas_policy_loss", dict(x=A, ld=16, ids=A, adv=A, old=A, ref=A, w=A, T=4, V=10, scale=1.0, reduce=1.0, low=0.2, high=0.2, kl=0.1,
                                            flags=0, logp=A, d=2 * A, ldo=16, stats=A, **WS), **kw)


@pytest.mark.parametrize("call", [_fwd, _bwd, _loss, _policy])
def test_refusals_on_logits(call):
    assert call(flags=2) == FLAGS and call(flags=8) == FLAGS
    for T in (-1, 1 << 31, 2 ** 63 - 1):
        assert call(T=T) == SHAPE
    for V in (0, -5, (1 << 30) + 1, 2 ** 63 - 1):
        assert call(V=V) == SHAPE
    for ld in (9, 0, -16, (1 << 31) + 1):
        assert call(ld=ld) == SHAPE
    for scale in (0.0, -1.0, INF, NAN, 2.0 ** 101):
        assert call(scale=scale) == SHAPE
    assert call(x=None) == NULL and call(x=A + 1) == ALIGN and call(x=A + 2, flags=elas.ELAS_LOGITS_F32) == ALIGN
    assert call(ids=None) == NULL and call(ids=A + 2) == ALIGN and call(ids=A + 4, flags=elas.ELAS_IDS_I64) == ALIGN
    assert b"ids" in elas.lib().elas_last_error()


@pytest.mark.parametrize("call", [_bwd, _loss, _policy])
def test_refusals_of_gradients(call):
    assert call(ldo=9) == SHAPE and call(ldo=-1) == SHAPE and call(d=A + 1) == ALIGN
    assert call(d=A, ldo=17) == SHAPE               # in place with another pitch
    assert call(d=A + 2, flags=elas.ELAS_LOGITS_F32) == ALIGN


@pytest.mark.parametrize("call", [_loss, _policy])
def test_refusals_of_workspaces(call):
    assert call(wsb=elas.elas_token_loss_workspace_bytes(4, 10) - 1) == WORKSPACE
    assert call(ws=None) == NULL and call(ws=A + 8) == ALIGN


def test_other_refusals_on_logits():
    assert _fwd(logp=None) == NULL and _fwd(logp=A + 2) == ALIGN and _fwd(lse=A + 1) == ALIGN
    assert _bwd(d=None) == NULL and _bwd(dlogp=None) == NULL and _bwd(lse=None) == NULL and _bwd(dlse=A + 2) == ALIGN
    for call in (_loss, _policy):
        assert call(stats=None) == NULL and call(stats=A + 2) == ALIGN and call(w=A + 1) == ALIGN and call(logp=A + 3) == ALIGN
        assert call(reduce=NAN) == SHAPE and call(reduce=INF) == SHAPE
    assert _loss(z=NAN) == SHAPE and _loss(lse=A + 1) == ALIGN
    assert _policy(adv=None) == NULL and _policy(adv=A + 1) == ALIGN and _policy(old=A + 2) == ALIGN and _policy(ref=A + 2) == ALIGN
    assert _policy(ref=None) == NULL                # with a kl_coef
    assert _policy(kl=INF) == SHAPE
    for bad in (-0.1, 1.5, NAN):
        assert _policy(low=bad) == SHAPE
    for bad in (-0.1, NAN):
        assert _policy(high=bad) == SHAPE
    # without tokens nothing is inspected or launched where there are no statistics
    empty = dict(T=0, x=None, ids=None)
    assert _fwd(**empty, logp=None, lse=None) == 0
    assert _bwd(**empty, dlogp=None, dlse=None, lse=None, d=None, ldo=0) == 0


def test_preference_refusals():
    def call(**kw):
        return _status("elas_preference_loss", dict(logp=A, ref=A, off=A, N=5000, pairs=300, beta=0.1, smoothing=0.0, flags=0, margin=A, d=A, stats=A, **WS), **kw)

    assert call(flags=1) == FLAGS
    for bad in (-1, 1 << 30):
        assert call(pairs=bad) == SHAPE
    for bad in (-1, 1 << 40):
        assert call(N=bad) == SHAPE
    assert call(beta=NAN) == SHAPE and call(beta=INF) == SHAPE
    for bad in (-0.1, 1.1, NAN):
        assert call(smoothing=bad) == SHAPE
    assert call(off=None) == NULL and call(off=A + 2) == ALIGN and call(off=A + 4, flags=elas.ELAS_IDS_I64) == ALIGN
    assert call(logp=None) == NULL and call(ref=A + 1) == ALIGN and call(margin=A + 2) == ALIGN and call(d=A + 2) == ALIGN
    assert call(stats=None) == NULL and call(wsb=elas.elas_preference_loss_workspace_bytes(5000, 300) - 1) == WORKSPACE and call(ws=None) == NULL


def test_adamw_refusals():
    p = (ctypes.c_void_p * 2)(A, A + 4)
    n, t, w = (ctypes.c_int64 * 2)(5, 7), (ctypes.c_int32 * 2)(0, 0), (ctypes.c_float * 2)(0.0, 0.1)

    def call(**kw):
        return _status("elas_adamw_step", dict(p=p, g=p, c=None, n=n, pt=t, gt=t, w=w, count=2, bits=32, m=A, ms=None, v=A, vs=None, step=A, rate=1e-3,
                                               factor=None, b1=0.9, b2=0.99, eps=1e-8, norm=None, max=1.0, **WS), **kw)

    assert call(count=-1) == SHAPE and call(count=1 << 20) == SHAPE and call(bits=16) == SHAPE
    for k in ("p", "g", "n", "pt", "gt", "w"):
        assert call(**{k: None}) == NULL
    assert call(pt=(ctypes.c_int32 * 2)(0, 3)) == FLAGS and call(gt=(ctypes.c_int32 * 2)(-1, 0)) == FLAGS
    assert call(n=(ctypes.c_int64 * 2)(5, -1)) == SHAPE and call(n=(ctypes.c_int64 * 2)(5, 1 << 40)) == SHAPE
    assert call(w=(ctypes.c_float * 2)(0.0, NAN)) == SHAPE
    for k in ("p", "g"):
        assert call(**{k: (ctypes.c_void_p * 2)(A, None)}) == NULL and call(**{k: (ctypes.c_void_p * 2)(A, A + 2)}) == ALIGN
    assert call(p=(ctypes.c_void_p * 2)(A, A + 2), pt=(ctypes.c_int32 * 2)(0, 1), ws=None) == NULL       # (bf16: 2 bytes are enough)
    assert call(c=(ctypes.c_void_p * 2)(A, A + 1)) == ALIGN
    for k in ("m", "v"):
        assert call(**{k: None}) == NULL and call(**{k: A + 8}) == ALIGN
    assert call(ms=A) == FLAGS and call(vs=A) == FLAGS and call(bits=8, ms=A) == NULL and call(bits=8, vs=A) == NULL
    for bad in (1.0, -0.1, NAN, 1 - 1e-9):          # (the last is 1 in float32)
        assert call(b1=bad) == SHAPE and call(b2=bad) == SHAPE
    for bad in (0.0, -1.0, NAN, INF, 1e-60, 1e60):
        assert call(eps=bad) == SHAPE
    assert call(rate=NAN) == SHAPE and call(rate=1e300) == SHAPE and call(max=-1.0) == SHAPE and call(max=NAN) == SHAPE
    assert call(step=None) == NULL and call(step=A + 4) == ALIGN and call(norm=A + 2) == ALIGN and call(factor=A + 1) == ALIGN
    assert call(ws=None) == NULL and call(ws=A + 8) == ALIGN and call(wsb=elas.elas_adamw_workspace_bytes() - 1) == WORKSPACE


def test_adamw_refuses_an_eps_without_a_reciprocal():
    """0 / (0 + eps) is 0 only where 1 / eps is a float32."""
    def call(eps):
        p, n, t, w = (ctypes.c_void_p * 1)(A), (ctypes.c_int64 * 1)(5), (ctypes.c_int32 * 1)(0), (ctypes.c_float * 1)(0.0)
        # (no workspace: an eps that is taken is refused for that)
        return _status("elas_adamw_step", dict(p=p, g=p, c=None, n=n, pt=t, gt=t, w=w, count=1, bits=32, m=A, ms=None, v=A, vs=None, step=A, rate=1e-3,
                                               factor=None, b1=0.9, b2=0.99, eps=eps, norm=None, max=1.0, **dict(WS, ws=None)))

    assert call(1e-40) == SHAPE and call(2.0 ** -127) == SHAPE and call(2.0 ** -126) == NULL


def test_adam8_values_refusals():
    def call(**kw):
        return _status("elas_adam8_values", dict(codes=A, scale=A, blocks=4, flags=0, out=A), **kw)

    assert call(flags=4) == FLAGS and call(blocks=-1) == SHAPE and call(blocks=1 << 32) == SHAPE
    for k in ("codes", "scale", "out"):
        assert call(**{k: None}) == NULL and call(**{k: A + 8}) == ALIGN
    assert call(blocks=0, codes=None, scale=None, out=None) == 0


def test_workspace_of_sizes_out_of_range():
    big = 2 ** 63 - 1
    for T, V in ((big, 10), (1 << 31, 10), (-1, 10), (4, 0), (4, big), (4, (1 << 30) + 1)):
        assert elas.elas_token_loss_workspace_bytes(T, V) == 0
    for N, pairs in ((100, -1), (100, 1 << 30), (100, big), (-1, 100), (1 << 40, 100)):
        assert elas.elas_preference_loss_workspace_bytes(N, pairs) == 0
    assert elas.elas_preference_loss_workspace_bytes(1000, 8) == 0 and elas.elas_preference_loss_workspace_bytes(1 << 20, 8) > 0
    # the largest that are taken: sums of workgroups, which do not grow with the tokens
    assert 0 < elas.elas_token_loss_workspace_bytes((1 << 31) - 1, 1 << 30) < 1 << 24
    assert 0 < elas.elas_preference_loss_workspace_bytes((1 << 40) - 1, (1 << 30) - 1) < 1 << 24


@pytest.mark.parametrize("flags", [0, elas.ELAS_LOGITS_F32])
@pytest.mark.parametrize("V", [1000, 8192, 32000, 131072])
def test_the_workspace_of_a_batch_is_enough_for_smaller_ones(V, flags):
    sizes = [elas.lib().elas_token_loss_workspace_bytes(T, V, flags) for T in range(1200)]
    assert sizes[0] == 0 and sizes == sorted(sizes)


def test_binding_refusals():
    """The binding's checks raise before any address is used; the tensors are on the CPU."""
    def raises(match, fn, *a, **k):
        with pytest.raises(ValueError, match=match):
            fn(*a, **k)

    x, ids = torch.zeros(4, 10, dtype=BF), torch.zeros(4, dtype=torch.int64)
    for fn in (lambda *a: elas.elas_token_logp_fwd(*a), lambda *a: elas.elas_token_loss(*a),
               lambda *a: elas.elas_policy_loss(*a, torch.zeros(4)), lambda *a: elas.elas_token_logp_bwd(torch.zeros(4), *a, torch.zeros(4))):
        raises("logits must be a GPU", fn, x, ids)
        raises("logits must be 2-D", fn, x[0], ids)
        raises("logits must be torch", fn, x.half(), ids)
    raises("logp must be 1-D", elas.elas_preference_loss, x, ids)
    raises("logp must be 1-D", elas.elas_preference_loss, torch.zeros(8), torch.zeros(4, dtype=torch.int32))
    raises("offsets must be", elas.elas_preference_loss, torch.zeros(8), torch.zeros(3))
    raises("GPU", elas.elas_preference_loss, torch.zeros(8), torch.zeros(3, dtype=torch.int32))
    raises("bits", elas.ElasAdamW, [torch.zeros(4)], bits=16)
    raises("GPU", elas.ElasAdamW, [torch.zeros(4)])
    raises("out must be", elas.elas_adam8_values, torch.zeros(256, dtype=torch.uint8), torch.zeros(1), dtype=torch.float16)
    raises("GPU", elas.elas_adam8_values, torch.zeros(256, dtype=torch.uint8), torch.zeros(1))


class _OnGpu(torch.Tensor):
    """Values that call themselves a tensor on GPU 0."""

    def get_device(self):
        return 0


def test_pitches():
    """Rows may have any pitch that keeps them apart."""
    def matrix(t):
        return binding._matrix(t.as_subclass(_OnGpu), t.shape, BF, 0, "x")[1]

    full = torch.zeros(6, 20, dtype=BF)
    assert matrix(full) == 20 and matrix(full[:, 3:11]) == 20 and matrix(full[::2, :7]) == 40
    assert matrix(full[:1].expand(1, 20)) == 20 and matrix(full[:, :1]) == 20 and matrix(full[:0]) == 20
    assert matrix(full[2:3, 4:9]) == 5                 # one row: its length
    for bad in (full.t(), full[:, ::2], full[:1].expand(6, 20), full.as_strided((4, 10), (5, 1))):
        with pytest.raises(ValueError, match="contiguous rows"):
            matrix(bad)


def test_gradients_beside_their_logits():
    """dlogits is logits itself, apart from it, or other columns of rows of one pitch."""
    buf = torch.zeros(400, dtype=BF)
    rows = lambda at, pitch, n=4, v=8: buf[at:].as_strided((n, v), (pitch, 1))  # noqa: E731
    x = rows(40, 24)
    def apart(d, x):
        (n, v), at = x.shape, lambda t: (t.data_ptr(), t.stride(0))  # noqa: E731
        binding._apart(n, v, 2, *at(x), *at(d))

    for good in (rows(40, 24), rows(48, 24), rows(32, 24), rows(56, 24), rows(40 + 3 * 24 + 8, 10), rows(0, 8), torch.zeros(4, 8, dtype=BF)):
        apart(good, x)
    for bad in (rows(41, 24), rows(47, 24), rows(33, 24), rows(57, 24), rows(40, 16), rows(16, 8), rows(40 + 24, 24)):
        with pytest.raises(ValueError, match="overlap"):
            apart(bad, x)
    apart(x[:0], x[:0])


def test_results_apart_from_operands():
    """A policy loss whose logp goes over old_logp (which other waves may still read), and the like, is refused
    before the call."""
    gpu = lambda t: t.as_subclass(_OnGpu)  # noqa: E731
    x, ids, rows = gpu(torch.zeros(4, 10)), gpu(torch.zeros(4, dtype=torch.int64)), gpu(torch.zeros(60))
    row = lambda k, shift=0: rows[8 * k + shift:8 * k + shift + 4]  # noqa: E731
    stats = {"stats": rows[50:52]}
    for fn, a, k in ((elas.elas_token_logp_fwd, (), {"out": {"logp": row(0), "lse": row(0)}}),
                     (elas.elas_token_logp_fwd, (), {"out": {"logp": row(0), "lse": row(0, 3)}}),
                     (elas.elas_token_loss, (), {"out": {**stats, "logp": row(0), "lse": row(0, 1)}}),
                     (elas.elas_token_loss, (row(1),), {"out": {**stats, "logp": row(1)}}),
                     (elas.elas_token_loss, (row(1),), {"out": {**stats, "lse": row(1, -3)}}),
                     *((elas.elas_policy_loss, (row(1), row(2), row(3), row(4)), {"out": {"stats": rows[50:53], "logp": row(j)}}) for j in range(1, 5))):
        with pytest.raises(ValueError, match="overlap"):
            fn(x, ids, *a, **k)
    binding._rows_apart(4, (100, 116), (84, 132, None))
    binding._rows_apart(4, (100, None), (None, 200))
    binding._rows_apart(0, (100, 100), (100,))


def test_calls_go_to_the_operands_gpu(monkeypatch):
    """A default stream's handle does not say which GPU it is of: a call for another GPU than
    the current one is made with that one current."""
    current, seen = [0], []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, current[0] = current[0], self.index

        def __exit__(self, *a):
            current[0] = self.before

    monkeypatch.setattr(binding, "_current", lambda: current[0])
    monkeypatch.setattr(binding, "_stream", lambda d: 100 + d)
    monkeypatch.setattr(torch.cuda, "device", Device)
    for device in (0, 1, 0):
        binding._on(device, lambda *a: seen.append((current[0], a)) or 0, 7)
    assert seen == [(0, (7, 100)), (1, (7, 101)), (0, (7, 100))] and current == [0]
