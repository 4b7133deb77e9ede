"""The entry points of include/elas_train.h on the host: exported, and refusing
every invalid argument with its status before anything is launched (so these
calls never touch a GPU); the binding's checks of shapes, types and devices."""
import ctypes
import os
import re

import pytest
import torch

import paper_2605_03667_amd as elas

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "elas_train.h")

pytestmark = pytest.mark.skipif(not os.path.exists(elas.LIB_PATH), reason="libelas.so not built")

A = 0x10000            # aligned, never dereferenced: every call below fails validation
MIS = 0x10008
NULL, SHAPE, ALIGN, WORKSPACE, FLAGS = 1, 2, 3, 4, 5
BF, F32 = torch.bfloat16, torch.float32


def test_exports_and_constants():
    text = open(HEADER).read()
    names = set(re.findall(r"\b(elas_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert len(names) == 9 and names <= set(elas._SIGNATURES)
    handle = ctypes.CDLL(elas.LIB_PATH)
    assert all(hasattr(handle, n) for n in names)
    defines = dict(re.findall(r"#define\s+(ELAS_[A-Z0-9_]+)\s+([0-9]+)u?", text))
    assert len(defines) == 6
    for k, v in defines.items():
        assert getattr(elas, k) == int(v), k
    assert set(elas.train.__all__) <= set(elas.__all__)


def _fwd(**kw):
    a = dict(h=A, b=A, gate=A, w_post=A, w_pre=A, T=4, d=16, rs=1.0, bs=1.0, eps=1e-6, flags=0, ho=A, n=A)
    a.update(kw)
    return elas.lib().elas_norm_join_fwd(*a.values(), None)


def test_norm_join_fwd_refusals():
    assert _fwd(flags=4) == FLAGS
    for bad in (0, 12, -8, 65544):
        assert _fwd(d=bad) == SHAPE
    assert _fwd(T=-1) == SHAPE and _fwd(T=1 << 31) == SHAPE
    for k in ("rs", "bs", "eps"):
        assert _fwd(**{k: float("inf")}) == SHAPE and _fwd(**{k: float("nan")}) == SHAPE
    assert _fwd(eps=-1.0) == SHAPE
    for k in ("h", "ho", "n"):
        assert _fwd(**{k: None}) == NULL and _fwd(**{k: MIS}) == ALIGN
    for k in ("b", "gate", "w_post", "w_pre"):
        assert _fwd(**{k: MIS}) == ALIGN
    # operands without the block they belong to, outputs without their operand
    assert _fwd(b=None) == FLAGS
    assert _fwd(b=None, gate=None) == FLAGS
    assert _fwd(b=None, gate=None, w_post=None) == FLAGS          # h_out
    assert _fwd(b=None, gate=None, w_post=None, ho=None, w_pre=None) == NULL
    assert _fwd(w_pre=None) == FLAGS                              # n
    assert _fwd(gate=None, flags=elas.ELAS_GATE_TOKEN) == NULL
    assert b"gate" in elas.lib().elas_last_error()
    assert _fwd(T=0, **dict.fromkeys(("h", "b", "gate", "w_post", "w_pre", "ho", "n"))) == 0


def _bwd(**kw):
    T, d = kw.get("T", 4), kw.get("d", 16)
    need = elas.elas_norm_join_bwd_workspace_bytes(max(T, 0), max(d, 8), 0)
    a = dict(dho=A, dn=A, ho=A, b=A, gate=A, w_post=A, w_pre=A, T=4, d=16, rs=1.0, bs=1.0, eps=1e-6, flags=0, dh=A, db=A, dgate=A,
             dpost=A, dpre=A, ws=A, wsb=need)
    a.update(kw)
    return elas.lib().elas_norm_join_bwd(*a.values(), None)


def test_norm_join_bwd_refusals():
    assert _bwd(flags=8) == FLAGS and _bwd(d=20) == SHAPE and _bwd(T=-2) == SHAPE and _bwd(eps=-1.0) == SHAPE
    for k in ("dn", "ho", "db", "dgate", "dpost", "dpre"):
        assert _bwd(**{k: None}) == NULL and _bwd(**{k: MIS}) == ALIGN
    for k in ("dho", "dh", "b", "gate", "w_post", "w_pre", "ws"):
        assert _bwd(**{k: MIS}) == ALIGN
    assert _bwd(w_pre=None) == FLAGS and _bwd(w_pre=None, dn=None) == FLAGS
    assert _bwd(w_pre=None, dn=None, dpre=None, dho=None) == NULL
    assert _bwd(gate=None) == FLAGS and _bwd(w_post=None) == FLAGS
    assert _bwd(b=None, gate=None, w_post=None, dgate=None, dpost=None) == FLAGS    # db
    assert _bwd(wsb=0) == WORKSPACE and _bwd(ws=None) == NULL
    assert _bwd(flags=elas.ELAS_GATE_TOKEN, gate=None) == NULL


def test_embed_refusals():
    def fwd(**kw):
        a = dict(ids=A, table=A, T=4, V=10, d=16, scale=1.0, flags=0, x=A)
        a.update(kw)
        return elas.lib().elas_embed_fwd(*a.values(), None)

    assert fwd(flags=2) == FLAGS and fwd(flags=8) == FLAGS
    assert fwd(T=-1) == SHAPE and fwd(V=0) == SHAPE and fwd(V=1 << 31) == SHAPE and fwd(d=4) == SHAPE
    assert fwd(scale=float("nan")) == SHAPE
    assert fwd(ids=None) == NULL and fwd(table=None) == NULL and fwd(x=MIS) == ALIGN and fwd(ids=A + 2) == ALIGN
    assert fwd(flags=elas.ELAS_IDS_I64, ids=A + 4) == ALIGN
    assert fwd(T=0, ids=None, table=None, x=None) == 0

    def bwd(**kw):
        a = dict(ids=A, dx=A, T=5000, V=10, d=16, scale=1.0, flags=0, dtable=A, ws=A, wsb=elas.elas_embed_bwd_workspace_bytes(5000, 10, 16, 0))
        a.update(kw)
        return elas.lib().elas_embed_bwd(*a.values(), None)

    assert bwd(flags=2) == FLAGS and bwd(V=-1) == SHAPE and bwd(dx=None) == NULL and bwd(dtable=None) == NULL
    assert bwd(dtable=MIS) == ALIGN and bwd(wsb=1) == WORKSPACE and bwd(ws=None) == NULL
    assert bwd(T=0, flags=elas.ELAS_EMBED_ADD, ids=None, dx=None, dtable=None, ws=None, wsb=0) == 0


def test_grad_refusals():
    p = (ctypes.c_void_p * 2)(A, A + 4)
    n = (ctypes.c_int64 * 2)(5, 7)
    t = (ctypes.c_int32 * 2)(0, 0)
    need = elas.elas_grad_workspace_bytes(2)
    L = elas.lib()

    def clip(grads=p, out=None, numel=n, dtype=t, count=2, max_norm=1.0, stats=A, ws=A, wsb=need):
        return L.elas_grad_clip(grads, out, numel, dtype, count, max_norm, stats, ws, wsb, None)

    assert clip(count=-1) == SHAPE and clip(count=1 << 20) == SHAPE
    assert clip(grads=None) == NULL and clip(numel=None) == NULL and clip(dtype=None) == NULL
    assert clip(dtype=(ctypes.c_int32 * 2)(0, 2)) == FLAGS
    assert clip(numel=(ctypes.c_int64 * 2)(5, -1)) == SHAPE and clip(numel=(ctypes.c_int64 * 2)(5, 1 << 44)) == SHAPE
    assert clip(grads=(ctypes.c_void_p * 2)(A, None)) == NULL and clip(grads=(ctypes.c_void_p * 2)(A, A + 2)) == ALIGN
    assert clip(out=(ctypes.c_void_p * 2)(A, A + 1)) == ALIGN and clip(out=(ctypes.c_void_p * 2)(A, None)) == NULL
    assert clip(max_norm=-1.0) == SHAPE and clip(max_norm=float("nan")) == SHAPE
    assert clip(stats=None) == NULL and clip(stats=A + 2) == ALIGN
    assert clip(wsb=need - 1) == WORKSPACE and clip(ws=None) == NULL and clip(ws=MIS) == ALIGN
    assert L.elas_grad_norm(p, n, t, 2, None, A, need, None) == NULL


def test_binding_refusals():
    """The binding's checks raise before any address is used; the tensors are on the CPU."""
    T, d = 4, 16
    h, b, g = torch.zeros(T, d, dtype=BF), torch.zeros(T, d, dtype=BF), torch.zeros(d, dtype=BF)

    def raises(match, fn, *a, **k):
        with pytest.raises(ValueError, match=match):
            fn(*a, **k)

    fwd, bwd = elas.elas_norm_join_fwd, elas.elas_norm_join_bwd
    raises("GPU", fwd, h, b, w_pre=g)
    raises("h must be", fwd, h.half(), b)
    raises("contiguous", fwd, torch.zeros(d, T, dtype=BF).t(), b)
    raises("dh", bwd, None, None, None)
    raises("table", elas.elas_embed_fwd, torch.zeros(3, dtype=torch.int32), g)
    raises("ids", elas.elas_embed_fwd, torch.zeros(3), torch.zeros(4, d, dtype=BF))
    raises("ids", elas.elas_embed_bwd, torch.zeros(3), torch.zeros(3, d, dtype=BF), 4)
    raises("GPU", elas.elas_embed_bwd, torch.zeros(3, dtype=torch.int32), torch.zeros(3, d, dtype=BF), 4)
    raises("GPU", elas.elas_grad_norm, [torch.zeros(3)])
    raises("tensor 0 must be", elas.elas_grad_clip, [torch.zeros(3, dtype=torch.float64)], 1.0)


@pytest.mark.gpu
def test_binding_refusals_on_the_gpu():
    """Shapes, types and devices that would make a kernel read past a buffer."""
    T, d, dev = 4, 16, "cuda:0"
    h, b, g = (torch.zeros(s, dtype=BF, device=dev) for s in ((T, d), (T, d), (d,)))

    def raises(match, fn, *a, **k):
        with pytest.raises(ValueError, match=match):
            fn(*a, **k)

    fwd, bwd = elas.elas_norm_join_fwd, elas.elas_norm_join_bwd
    raises("b has shape", fwd, h, b[:3], w_pre=g)
    raises("gate has shape", fwd, h, b, gate=torch.zeros(T + 1, d, dtype=BF, device=dev))
    raises("w_pre has shape", fwd, h, w_pre=torch.zeros(d + 8, dtype=BF, device=dev))
    raises("w_post must be", fwd, h, b, w_post=g.float())
    raises("b must be a GPU", fwd, h, b.cpu())
    raises("contiguous", fwd, h, torch.zeros(T, 2 * d, dtype=BF, device=dev)[:, :d])
    raises("out\\['n'\\]", fwd, h, b, w_pre=g, out={"h": h.clone()})
    raises("out\\['h'\\]", fwd, h, b, out={"h": h.float()})
    raises("dn is given", bwd, h, h, h, b)
    raises("dn is required", bwd, h, None, h, b, w_pre=g)
    raises("h must be", bwd, h, h, h.float(), w_pre=g)
    raises("dw_pre", bwd, h, h, h, w_pre=g, grads={"dh": h.clone(), "dw_pre": g})
    ids = torch.zeros(T, dtype=torch.int32, device=dev)
    raises("dx has shape", elas.elas_embed_bwd, ids, h[:3], 5)
    raises("dtable is required", elas.elas_embed_bwd, ids, h, 5, accumulate=True)
    raises("dtable has shape", elas.elas_embed_bwd, ids, h, 5, dtable=torch.zeros(4, d, device=dev))
    raises("out has shape", elas.elas_embed_fwd, ids, h, out=h[:3])
    raises("dtype", elas.elas_embed_fwd, ids, h, dtype=torch.float16)
    x = torch.zeros(8, device=dev)
    raises("types, lengths", elas.elas_grad_clip, [x], 1.0, out=[x[:4]])
    raises("types, lengths", elas.elas_grad_clip, [x], 1.0, out=[x.to(BF)])
    raises("contiguous", elas.elas_grad_norm, [x[::2]])
    raises("stats", elas.elas_grad_clip, [x], 1.0, stats=x)
    with pytest.raises(elas.ElasError, match="multiple of 8"):
        fwd(torch.zeros(2, 12, dtype=BF, device=dev), w_pre=torch.zeros(12, dtype=BF, device=dev))
    with pytest.raises(elas.ElasError, match="WORKSPACE"):
        bwd(h, h, h, w_pre=g, workspace=torch.zeros(16, dtype=torch.uint8, device=dev))
