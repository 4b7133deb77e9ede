"""Binding of the operators around the FFN in a training step (the C ABI of
``include/elas_train.h``): the norms before and after a block with its gate and
residual scale, the embedding, and the norm and clipping of the gradients.

As in the package's other functions, every step runs in the HIP kernels of
``libelas.so``; the functions check sizes, types and devices, allocate what is
not passed in, and take the current stream.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from . import _check, _f32, _i64, _p, _SIGNATURES, _sz, _u32, _workspace, lib

__all__ = [
    "ELAS_RES_F32", "ELAS_GATE_TOKEN", "ELAS_IDS_I64", "ELAS_EMBED_ADD", "ELAS_GRAD_F32", "ELAS_GRAD_BF16",
    "elas_norm_join_fwd", "elas_norm_join_bwd", "elas_norm_join_bwd_workspace_bytes", "elas_embed_fwd", "elas_embed_bwd",
    "elas_embed_bwd_workspace_bytes", "ElasTensors", "elas_grad_norm", "elas_grad_clip", "elas_grad_workspace_bytes",
]

ELAS_RES_F32 = 1
ELAS_GATE_TOKEN = 2
ELAS_IDS_I64 = 4
ELAS_EMBED_ADD = 8
ELAS_GRAD_F32 = 0
ELAS_GRAD_BF16 = 1

_pp = ctypes.POINTER(_p)
_i64p = ctypes.POINTER(_i64)
_i32p = ctypes.POINTER(ctypes.c_int32)
_SIGNATURES.update({
    "elas_norm_join_fwd": ([_p] * 5 + [_i64] * 2 + [_f32] * 3 + [_u32] + [_p] * 3, ctypes.c_int),
    "elas_norm_join_bwd_workspace_bytes": ([_i64, _i64, _u32], _sz),
    "elas_norm_join_bwd": ([_p] * 7 + [_i64] * 2 + [_f32] * 3 + [_u32] + [_p] * 5 + [_p, _sz, _p], ctypes.c_int),
    "elas_embed_fwd": ([_p] * 2 + [_i64] * 3 + [_f32, _u32] + [_p] * 2, ctypes.c_int),
    "elas_embed_bwd_workspace_bytes": ([_i64, _i64, _i64, _u32], _sz),
    "elas_embed_bwd": ([_p] * 2 + [_i64] * 3 + [_f32, _u32] + [_p, _p, _sz, _p], ctypes.c_int),
    "elas_grad_workspace_bytes": ([_i64], _sz),
    "elas_grad_norm": ([_pp, _i64p, _i32p, _i64, _p, _p, _sz, _p], ctypes.c_int),
    "elas_grad_clip": ([_pp, _pp, _i64p, _i32p, _i64, _f32, _p, _p, _sz, _p], ctypes.c_int),
})

_BF16, _F32 = torch.bfloat16, torch.float32


# torch's current stream of a device, without the object that torch.cuda.current_stream makes
# (0.1 us instead of 1.9, of calls of 6)
_stream = torch._C._cuda_getCurrentRawStream


def _arg(t: torch.Tensor, shape, dtype: torch.dtype, device: int, name: str) -> int:
    """Address of tensor ``t``, which must have exactly this shape and type, be
    contiguous and lie on GPU ``device`` (the C ABI gets a bare address)."""
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.get_device() != device or device < 0:
        raise ValueError(f"{name} must be a GPU tensor" + (f" on device {device}" if device >= 0 else ""))
    return t.data_ptr()


def _opt(t, shape, dtype, device, name):
    return None if t is None else _arg(t, shape, dtype, device, name)


def _required(t, name):
    if t is None:
        raise ValueError(f"{name} is required")
    return t


def _scratch(workspace, need: int, device: torch.device):
    """The caller's workspace (bytes, on the operands' GPU ``device``) or a new one:
    the tensor, its address and size."""
    if workspace is None:
        workspace = _workspace(need, device)
    if workspace is None:
        return None, None, 0
    return workspace, _arg(workspace, (workspace.numel(),), torch.uint8, device.index, "workspace"), workspace.numel()


def _res_flag(dtype: torch.dtype, name: str) -> int:
    if dtype == _BF16:
        return 0
    if dtype == _F32:
        return ELAS_RES_F32
    raise ValueError(f"{name} must be torch.bfloat16 or torch.float32, got {dtype}")


# ---- norms before and after a block ------------------------------------------------


def _join_operands(T, d, dev, b, gate, w_post, w_pre):
    """Addresses of the operands both directions share, and the gate's flag."""
    row = (d,)
    token = gate is not None and gate.dim() == 2
    return (_opt(b, (T, d), _BF16, dev, "b"), _opt(gate, (T, d) if token else row, _BF16, dev, "gate"),
            _opt(w_post, row, _BF16, dev, "w_post"), _opt(w_pre, row, _BF16, dev, "w_pre"), ELAS_GATE_TOKEN if token else 0)


def elas_norm_join_fwd(h, b=None, gate=None, w_post=None, w_pre=None, res_scale: float = 1.0, block_scale: float = 1.0,
                       eps: float = 1e-6, out: dict | None = None) -> dict:
    """Joins a block's output b [T, d] to the residual stream h [T, d] (bf16 or
    float32) and normalises the sum for the next block:

        h' = res_scale h + block_scale gate (norm(b) w_post),   n = norm(h') w_pre

    with norm(v) = v / sqrt(mean(v^2) + eps) over the features.  gate is [d]
    (shared by the tokens), [T, d] or None; without w_post b is not normalised;
    without w_pre there is no n; without b only n = norm(h) w_pre is computed.
    Returns dict(h, n), h being h' in h's type (None without b) and n bf16."""
    T, d = h.shape
    dev = h.get_device()
    flags = _res_flag(h.dtype, "h")
    h_p = _arg(h, (T, d), h.dtype, dev, "h")
    b_p, gate_p, post_p, pre_p, gate_flag = _join_operands(T, d, dev, b, gate, w_post, w_pre)
    if out is None:
        out = {"h": None if b is None else torch.empty_like(h),
               "n": None if w_pre is None else torch.empty((T, d), dtype=_BF16, device=h.device)}
    ho_p = None if b is None else _arg(_required(out.get("h"), "out['h']"), (T, d), h.dtype, dev, "out['h']")
    n_p = None if w_pre is None else _arg(_required(out.get("n"), "out['n']"), (T, d), _BF16, dev, "out['n']")
    _check(lib().elas_norm_join_fwd(h_p, b_p, gate_p, post_p, pre_p, T, d, res_scale, block_scale, eps, flags | gate_flag,
                                    ho_p, n_p, _stream(dev)))
    return out


@functools.lru_cache(maxsize=1024)   # (of the sizes alone)
def elas_norm_join_bwd_workspace_bytes(T: int, d: int, flags: int = 0) -> int:
    return lib().elas_norm_join_bwd_workspace_bytes(T, d, flags)


def elas_norm_join_bwd(dh, dn, h, b=None, gate=None, w_post=None, w_pre=None, res_scale: float = 1.0, block_scale: float = 1.0,
                       eps: float = 1e-6, grads: dict | None = None, workspace: torch.Tensor | None = None) -> dict:
    """Gradient of elas_norm_join_fwd.  dh [T, d] is the gradient of the joined
    stream h' from the rest of the network (None: zero), dn that of n, h the
    forward's h' (its input h where it had no b); the operands are the forward's.
    Returns dict(dh, db, dgate, dw_post, dw_pre), each None where its operand is:
    dh in the residual stream's type, db bf16, dgate bf16 [T, d] or float32 [d],
    the gains' gradients float32 [d]."""
    like = dh if dh is not None else _required(h, "h (or dh)")
    T, d = like.shape
    dev = like.get_device()
    res = like.dtype
    flags = _res_flag(res, "dh" if dh is not None else "h")
    rows, row = (T, d), (d,)
    dh_p = _opt(dh, rows, res, dev, "dh")
    dn_p = h_p = None
    if w_pre is not None:
        dn_p = _arg(_required(dn, "dn"), rows, _BF16, dev, "dn")
        h_p = _arg(_required(h, "h"), rows, res, dev, "h")
    elif dn is not None:
        raise ValueError("dn is given without w_pre")
    b_p, gate_p, post_p, pre_p, gate_flag = _join_operands(T, d, dev, b, gate, w_post, w_pre)
    device = like.device
    if grads is None:
        grads = {
            "dh": torch.empty(rows, dtype=res, device=device),
            "db": None if b is None else torch.empty(rows, dtype=_BF16, device=device),
            "dgate": None if gate is None else torch.empty(gate.shape, dtype=_BF16 if gate_flag else _F32, device=device),
            "dw_post": None if w_post is None else torch.empty(row, dtype=_F32, device=device),
            "dw_pre": None if w_pre is None else torch.empty(row, dtype=_F32, device=device),
        }

    def grad(key, operand, shape, dtype):
        return None if operand is None else _arg(_required(grads.get(key), key), shape, dtype, dev, key)

    out = (grad("dh", like, rows, res), grad("db", b, rows, _BF16),
           grad("dgate", gate, rows if gate_flag else row, _BF16 if gate_flag else _F32),
           grad("dw_post", w_post, row, _F32), grad("dw_pre", w_pre, row, _F32))
    workspace, ws_p, ws_n = _scratch(workspace, elas_norm_join_bwd_workspace_bytes(T, d, flags | gate_flag), device)
    _check(lib().elas_norm_join_bwd(dh_p, dn_p, h_p, b_p, gate_p, post_p, pre_p, T, d, res_scale, block_scale, eps,
                                    flags | gate_flag, *out, ws_p, ws_n, _stream(dev)))
    return grads


# ---- embedding -----------------------------------------------------------------------


def _ids(ids, dev):
    if ids.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"ids must be torch.int32 or torch.int64, got {ids.dtype}")
    return _arg(ids, ids.shape, ids.dtype, dev, "ids"), ELAS_IDS_I64 if ids.dtype == torch.int64 else 0


def elas_embed_fwd(ids, table, scale: float = 1.0, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None):
    """x[...] = scale * table[ids[...]] for ids of any shape (int32 or int64) and a
    bf16 table [V, d]; x [*ids.shape, d] is bf16 or float32.  An id outside
    0 .. V-1 gives a row of zeros."""
    if table.dim() != 2:
        raise ValueError("table must be 2-D")
    V, d = table.shape
    dev = table.get_device()
    ids_p, flags = _ids(ids, dev)
    if out is None:
        out = torch.empty((*ids.shape, d), dtype=dtype, device=table.device)
    flags |= _res_flag(dtype, "dtype")
    table_p = _arg(table, (V, d), _BF16, dev, "table")
    out_p = _arg(out, (*ids.shape, d), dtype, dev, "out")
    _check(lib().elas_embed_fwd(ids_p, table_p, ids.numel(), V, d, scale, flags, out_p, _stream(dev)))
    return out


@functools.lru_cache(maxsize=1024)   # (of the sizes alone)
def elas_embed_bwd_workspace_bytes(T: int, V: int, d: int, flags: int = 0) -> int:
    return lib().elas_embed_bwd_workspace_bytes(T, V, d, flags)


def elas_embed_bwd(ids, dx, V: int, scale: float = 1.0, dtable: torch.Tensor | None = None, accumulate: bool = False,
                   workspace: torch.Tensor | None = None):
    """Gradient of elas_embed_fwd: dtable [V, d] (float32), row v the sum of scale *
    dx over the tokens whose id is v; added to what ``dtable`` holds with
    ``accumulate`` (rows without tokens are then not touched).  dx [*ids.shape, d]
    is bf16 or float32.  The sums' order depends on the ids alone."""
    d = dx.shape[-1]
    dev = dx.get_device()
    ids_p, flags = _ids(ids, dev)
    flags |= _res_flag(dx.dtype, "dx")
    dx_p = _arg(dx, (*ids.shape, d), dx.dtype, dev, "dx")
    if accumulate:
        _required(dtable, "dtable")
        flags |= ELAS_EMBED_ADD
    elif dtable is None:
        dtable = torch.empty((V, d), dtype=_F32, device=dx.device)
    dtable_p = _arg(dtable, (V, d), _F32, dev, "dtable")
    T = ids.numel()
    workspace, ws_p, ws_n = _scratch(workspace, elas_embed_bwd_workspace_bytes(T, V, d, flags), dx.device)
    _check(lib().elas_embed_bwd(ids_p, dx_p, T, V, d, scale, flags, dtable_p, ws_p, ws_n, _stream(dev)))
    return dtable


# ---- norm and clipping of the gradients ------------------------------------------------


class ElasTensors:
    """A list of GPU tensors (float32 or bf16, contiguous, any shapes) as the C ABI
    takes it.  A program that uses the same tensors every step makes it once; the
    tensors are held, and their addresses, lengths, types and layouts are read again
    at every call (a tensor's ``data`` may have been replaced since)."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        n = len(self.tensors)
        self._pointers = (_p * n)()
        self._numel = (_i64 * n)()
        self._dtype = (ctypes.c_int32 * n)()
        self.layout = self._addresses = None
        self._apart = False
        self.device = self.tensors[0].device if n else torch.device("cuda", torch.cuda.current_device())

    def __len__(self):
        return len(self.tensors)

    def arrays(self, written: bool = False):
        """The host arrays of addresses, lengths and types; of tensors that the call
        writes, no two may overlap."""
        ts = self.tensors
        addresses, layout = list(map(torch.Tensor.data_ptr, ts)), (list(map(torch.Tensor.numel, ts)), [t.dtype for t in ts])
        if addresses != self._addresses or layout != self.layout or not all(map(torch.Tensor.is_contiguous, ts)):
            dev = self.device.index
            for k, t in enumerate(ts):
                if t.dtype != _F32 and t.dtype != _BF16:
                    raise ValueError(f"tensor {k} must be torch.float32 or torch.bfloat16, got {t.dtype}")
                _arg(t, t.shape, t.dtype, -1 if dev is None else dev, f"tensor {k}")
            self._pointers[:], self._numel[:] = addresses, layout[0]
            self._dtype[:] = [ELAS_GRAD_F32 if t == _F32 else ELAS_GRAD_BF16 for t in layout[1]]
            self.layout, self._addresses, self._apart = layout, addresses, False
        if written and not self._apart:
            spans = sorted((a, a + n * t.itemsize) for a, n, t in zip(addresses, *layout) if n)
            if any(end > start for (_, end), (start, _) in zip(spans, spans[1:])):
                raise ValueError("tensors that are written must not overlap (one of them given twice?)")
            self._apart = True
        return self._pointers, self._numel, self._dtype


def _tensors(t) -> ElasTensors:
    return t if isinstance(t, ElasTensors) else ElasTensors(t)


@functools.lru_cache(maxsize=1024)   # (of the sizes alone)
def elas_grad_workspace_bytes(n: int) -> int:
    return lib().elas_grad_workspace_bytes(n)


def elas_grad_norm(grads, norm: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Euclidean norm over all values of ``grads`` (a list of tensors or an
    ElasTensors): float32 [1] on the GPU."""
    grads = _tensors(grads)
    dev = grads.device
    pointers, numel, dtype = grads.arrays()
    if norm is None:
        norm = torch.empty(1, dtype=_F32, device=dev)
    norm_p = _arg(norm, (1,), _F32, dev.index, "norm")
    workspace, ws_p, ws_n = _scratch(workspace, elas_grad_workspace_bytes(len(grads)), dev)
    _check(lib().elas_grad_norm(pointers, numel, dtype, len(grads), norm_p, ws_p, ws_n, _stream(dev.index)))
    return norm


def elas_grad_clip(grads, max_norm: float, out=None, stats: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Scales ``grads`` (a list of tensors or an ElasTensors) by factor =
    min(1, max_norm / norm), in place or into the tensors ``out`` of the same types
    and lengths; no tensor that is written may overlap another.  Returns stats,
    float32 [2] on the GPU: norm and factor.  Where a value is not finite the factor
    is 0 and the values are passed on unscaled."""
    grads = _tensors(grads)
    dev = grads.device
    pointers, numel, dtype = grads.arrays(written=out is None)
    out_p = None
    if out is not None:
        out = _tensors(out)
        out_p = out.arrays(written=True)[0]
        if out.layout != grads.layout or out.device != dev:
            raise ValueError("out must hold tensors of the same types, lengths and device as grads")
    if stats is None:
        stats = torch.empty(2, dtype=_F32, device=dev)
    stats_p = _arg(stats, (2,), _F32, dev.index, "stats")
    workspace, ws_p, ws_n = _scratch(workspace, elas_grad_workspace_bytes(len(grads)), dev)
    _check(lib().elas_grad_clip(pointers, out_p, numel, dtype, len(grads), max_norm, stats_p, ws_p, ws_n, _stream(dev.index)))
    return stats
