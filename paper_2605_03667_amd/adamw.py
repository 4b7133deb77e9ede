"""Binding of the update of a training step (the C ABI of ``include/elas_adamw.h``):
AdamW over many tensors at once, with its moments in 32 or 8 bits, the clipping by the
gradients' norm folded in, and bf16 copies of the weights written in the same pass.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import _check, _f32, _i64, _p, _SIGNATURES, _sz, _u32, lib
from .loss import _on
from .train import _arg, _BF16, _F32, _i32p, _i64p, _opt, _pp, _scratch, _tensors, ELAS_RES_F32, ElasTensors

__all__ = ["ELAS_ADAMW_BLOCK", "ELAS_ADAM8_SECOND", "ElasAdamW", "elas_adamw_step", "elas_adamw_workspace_bytes", "elas_adam8_values"]

ELAS_ADAMW_BLOCK = 256
ELAS_ADAM8_SECOND = 2

_f64 = ctypes.c_double
_f32p = ctypes.POINTER(_f32)
_SIGNATURES.update({
    "elas_adamw_workspace_bytes": ([], _sz),
    "elas_adamw_step": ([_pp, _pp, _pp, _i64p, _i32p, _i32p, _f32p, _i64, ctypes.c_int, _p, _p, _p, _p, _p, _f64, _p, _f64, _f64, _f64, _p, _f64,
                         _p, _sz, _p], ctypes.c_int),
    "elas_adam8_values": ([_p, _p, _i64, _u32, _p, _p], ctypes.c_int),
})


class ElasAdamW:
    """The state of AdamW over a list of tensors: the parameters (float32 or bf16,
    contiguous, any shapes), their bf16 copies where there are any (one for each
    parameter, None for those without one), a weight decay for each (``decay``: set as a
    whole, also between steps), and the moments.

    ``bits`` is 32 or 8.  The moments ``m`` and ``v`` are flat tensors (float32, or
    uint8 codes with a float32 scale for each block of 256 in ``m_scale`` and
    ``v_scale``); tensor k's begin at value 256 * sum of ceil(numel / 256) over the
    tensors before it.  ``step`` is an int64 [1] on the GPU, so that a captured graph
    counts its steps.  These tensors are the whole state: a checkpoint saves them."""

    def __init__(self, params, copies=None, decay=0.0, bits: int = 32):
        if bits not in (8, 32):
            raise ValueError(f"bits must be 8 or 32, got {bits}")
        self.params = _tensors(params)
        n = len(self.params)
        self.params.arrays(written=True)
        copies = [None] * n if copies is None else list(copies.tensors if isinstance(copies, ElasTensors) else copies)
        if len(copies) != n:
            raise ValueError(f"{n} parameters, {len(copies)} copies")
        self.bits = bits
        self.decay = decay
        self._with_copy = [k for k, c in enumerate(copies) if c is not None]
        self.copies = ElasTensors([copies[k] for k in self._with_copy]) if self._with_copy else None
        self._copy_pointers = (_p * n)()
        self._copy_addresses = None
        self._layout = self.params.layout
        self._disjoint = None
        self.blocks = sum(-(-k // ELAS_ADAMW_BLOCK) for k in self._layout[0])
        device = self.params.device
        total = self.blocks * ELAS_ADAMW_BLOCK
        kind = torch.uint8 if bits == 8 else _F32
        self.m, self.v = (torch.zeros(total, dtype=kind, device=device) for _ in range(2))
        self.m_scale, self.v_scale = (torch.zeros(self.blocks, device=device) if bits == 8 else None for _ in range(2))
        self.step = torch.zeros(1, dtype=torch.int64, device=device)
        self._workspace = torch.empty(elas_adamw_workspace_bytes(), dtype=torch.uint8, device=device)
        self._check_copies()

    def __len__(self):
        return len(self.params)

    @property
    def decay(self) -> tuple:
        return self._decays

    @decay.setter
    def decay(self, decay) -> None:
        n = len(self.params)
        decay = tuple(float(d) for d in decay) if hasattr(decay, "__len__") else (float(decay),) * n
        if len(decay) != n:
            raise ValueError(f"{n} parameters, {len(decay)} decays")
        if not all(map(math.isfinite, decay)):
            raise ValueError("decay must be finite")
        self._decays, self._decay = decay, (_f32 * n)(*decay)

    def _check_copies(self):
        """The host array of the copies' addresses (None: there are none)."""
        if self.copies is None:
            return None
        pointers = self.copies.arrays(written=True)[0]
        if self.copies._addresses is not self._copy_addresses:
            lengths, types = self.copies.layout
            for k, n, t in zip(self._with_copy, lengths, types):
                if t != _BF16 or n != self._layout[0][k]:
                    raise ValueError(f"copy {k} must be torch.bfloat16 and as long as its parameter")
            if self.copies.device != self.params.device:
                raise ValueError("copies must be on the parameters' device")
            for j, k in enumerate(self._with_copy):
                self._copy_pointers[k] = pointers[j]
            self._copy_addresses = self.copies._addresses
        return self._copy_pointers

    def _check_apart(self, grads: ElasTensors) -> None:
        """Raises where a parameter or a copy overlaps another tensor of the step (what one
        thread writes another would read)."""
        seen = (self.params._addresses, grads._addresses, self.copies and self.copies._addresses)
        before = self._disjoint
        if before is not None and seen[0] is before[0] and seen[1] is before[1] and seen[2] is before[2]:
            return
        lists = [(self.params, True), (grads, False)] + ([(self.copies, True)] if self.copies else [])
        spans = sorted((a, a + n * t.itemsize, written) for tensors, written in lists for a, n, t in zip(tensors._addresses, *tensors.layout) if n)
        end = end_written = 0
        for start, stop, written in spans:
            if start < (end if written else end_written):
                raise ValueError("parameters, copies and gradients must not overlap")
            end = max(end, stop)
            if written:
                end_written = max(end_written, stop)
        self._disjoint = seen


def elas_adamw_workspace_bytes() -> int:
    return lib().elas_adamw_workspace_bytes()


def elas_adamw_step(opt: ElasAdamW, grads, rate: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                    norm: torch.Tensor | None = None, max_norm: float = math.inf, rate_factor: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None) -> ElasAdamW:
    """One step of AdamW over all tensors of ``opt``, in place:

        m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2,  t = step + 1
        p = (1 - lr decay) p - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)

    grads is a list of tensors or an ElasTensors of the parameters' lengths, float32
    or bf16 each.  With ``norm`` (float32 [1] on the GPU, as elas_grad_norm gives it)
    g' = g min(1, max_norm / norm), and where the norm is not finite the step is
    skipped: nothing changes, nor does ``opt.step``.  lr is rate, times rate_factor
    (float32 [1] on the GPU, a schedule that a captured graph can follow) where that is given.
    The workspace is the state's own unless one is passed in."""
    grads = _tensors(grads)
    n = len(opt)
    pointers, numel, types = opt.params.arrays(written=True)
    if opt.params.layout is not opt._layout:
        if opt.params.layout[0] != opt._layout[0]:
            raise ValueError("the parameters' lengths are not those that the state was made for")
        opt._layout = opt.params.layout
    copies = opt._check_copies()
    grad_pointers, _, grad_types = grads.arrays()
    if grads.layout[0] != opt._layout[0] or grads.device != opt.params.device:
        raise ValueError("grads must hold tensors of the parameters' lengths and device")
    opt._check_apart(grads)
    dev = opt.params.device.index
    total = opt.blocks * ELAS_ADAMW_BLOCK
    kind = torch.uint8 if opt.bits == 8 else _F32
    m, v = _arg(opt.m, (total,), kind, dev, "m"), _arg(opt.v, (total,), kind, dev, "v")
    scale = (opt.blocks,)
    m_scale = v_scale = None
    if opt.bits == 8:
        m_scale, v_scale = _arg(opt.m_scale, scale, _F32, dev, "m_scale"), _arg(opt.v_scale, scale, _F32, dev, "v_scale")
    workspace, ws_p, ws_n = _scratch(opt._workspace if workspace is None else workspace, 0, opt.params.device)
    _on(dev, lib().elas_adamw_step, pointers, grad_pointers, copies, numel, types, grad_types, opt._decay, n, opt.bits, m, m_scale, v, v_scale,
        _arg(opt.step, (1,), torch.int64, dev, "step"), rate, _opt(rate_factor, (1,), _F32, dev, "rate_factor"), beta1, beta2, eps,
        _opt(norm, (1,), _F32, dev, "norm"), max_norm, ws_p, ws_n)
    return opt


def elas_adam8_values(codes, scale, second: bool = False, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """What moments in 8 bits stand for: codes uint8 [256 blocks] and scale float32
    [blocks] of first moments (``second``: of second ones) as bf16 or float32 [256 blocks]."""
    blocks = scale.numel()
    dev = codes.get_device()
    if out is None:
        out = torch.empty(blocks * ELAS_ADAMW_BLOCK, dtype=dtype, device=codes.device)
    if out.dtype != _BF16 and out.dtype != _F32:
        raise ValueError(f"out must be torch.bfloat16 or torch.float32, got {out.dtype}")
    flags = (ELAS_ADAM8_SECOND if second else 0) | (ELAS_RES_F32 if out.dtype == _F32 else 0)
    shape = (blocks * ELAS_ADAMW_BLOCK,)
    _on(dev, lib().elas_adam8_values, _arg(codes, shape, torch.uint8, dev, "codes"), _arg(scale, (blocks,), _F32, dev, "scale"), blocks, flags,
        _arg(out, shape, out.dtype, dev, "out"))
    return out
