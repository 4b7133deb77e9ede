"""Binding of the losses of a training step (the C ABI of ``include/elas_loss.h``):
log-probabilities of tokens from logits with their gradient, the token loss, the
clipped policy loss and the preference loss, each with its gradient in one call.

As in the package's other functions, every step runs in the HIP kernels of
``libelas.so``; the functions check sizes, types and devices, allocate what is
not passed in, and take the current stream.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from . import _check, _f32, _i64, _p, _SIGNATURES, _sz, _u32, lib
from .train import _arg, _F32, _BF16, _ids, _opt, _required, _scratch, _stream, ELAS_IDS_I64

__all__ = [
    "ELAS_LOGITS_F32", "elas_token_logp_fwd", "elas_token_logp_bwd", "elas_token_loss", "elas_token_loss_workspace_bytes",
    "elas_policy_loss", "elas_preference_loss", "elas_preference_loss_workspace_bytes",
]

ELAS_LOGITS_F32 = 1

_SIGNATURES.update({
    "elas_token_loss_workspace_bytes": ([_i64, _i64, _u32], _sz),
    "elas_token_logp_fwd": ([_p, _i64, _p, _i64, _i64, _f32, _u32, _p, _p, _p], ctypes.c_int),
    "elas_token_logp_bwd": ([_p, _p, _p, _i64, _p, _p, _i64, _i64, _f32, _u32, _p, _i64, _p], ctypes.c_int),
    "elas_token_loss": ([_p, _i64, _p, _p, _i64, _i64, _f32, _f32, _f32, _u32, _p, _p, _p, _i64, _p, _p, _sz, _p], ctypes.c_int),
    "elas_policy_loss": ([_p, _i64, _p, _p, _p, _p, _p, _i64, _i64] + [_f32] * 5 + [_u32, _p, _p, _i64, _p, _p, _sz, _p], ctypes.c_int),
    "elas_preference_loss_workspace_bytes": ([_i64, _i64], _sz),
    "elas_preference_loss": ([_p, _p, _p, _i64, _i64, _f32, _f32, _u32, _p, _p, _p, _p, _sz, _p], ctypes.c_int),
})

# The GPU that calls go to by themselves.  A stream's handle of 0 (a GPU's default stream) does
# not say whose it is, so a call for another GPU is made with that one current.
_current = torch._C._cuda_getDevice


def _on(device: int, function, *args) -> None:
    """Calls the C function ``function`` with the arguments and the current stream of GPU ``device``."""
    if _current() == device:
        _check(function(*args, _stream(device)))
    else:
        with torch.cuda.device(device):
            _check(function(*args, _stream(device)))


def _matrix(t: torch.Tensor, shape, dtype: torch.dtype, device: int, name: str):
    """Address and pitch of a matrix whose rows are contiguous and do not overlap, on GPU
    ``device``; a single row's pitch is its length."""
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.get_device() != device or device < 0:
        raise ValueError(f"{name} must be a GPU tensor" + (f" on device {device}" if device >= 0 else ""))
    rows, columns = shape
    pitch, step = t.stride()
    if rows <= 1:
        pitch = columns
    if (step != 1 and columns > 1) or pitch < columns:
        raise ValueError(f"{name} must have contiguous rows that do not overlap, got strides {t.stride()}")
    return t.data_ptr(), pitch


def _logits(logits, ids):
    """(T, V, device, flags, logits' address and pitch, ids' address)."""
    shape = logits.shape
    if len(shape) != 2:
        raise ValueError(f"logits must be 2-D, got shape {tuple(shape)}")
    dtype = logits.dtype
    if dtype == _F32:
        flags = ELAS_LOGITS_F32
    elif dtype == _BF16:
        flags = 0
    else:
        raise ValueError(f"logits must be torch.bfloat16 or torch.float32, got {dtype}")
    dev = logits.get_device()
    x, ld = _matrix(logits, shape, dtype, dev, "logits")
    T, V = shape
    if ids.shape != shape[:1]:
        raise ValueError(f"ids has shape {tuple(ids.shape)}, expected {(T,)}")
    ids_p, ids_flag = _ids(ids, dev)
    return T, V, dev, flags | ids_flag, x, ld, ids_p


def _apart(T, V, size, x, ld, d, ld_out):
    """Raises where the memory of the gradient (at ``d``) overlaps the logits' (at ``x``) and is not the very same rows."""
    if d == x and ld_out == ld or not T:
        return
    end, end_out = x + ((T - 1) * ld + V) * size, d + ((T - 1) * ld_out + V) * size
    # (columns beside one another in rows of one pitch are apart)
    if x < end_out and d < end and (ld_out != ld or not V <= abs(x - d) // size % ld <= ld - V):
        raise ValueError("dlogits must be logits itself or overlap nothing of it")


def _gradient(dlogits, logits, dev, x, ld):
    """Address and pitch of the gradient's tensor; (None, 0) where it is not wanted."""
    if dlogits is None:
        return None, 0
    p, pitch = _matrix(dlogits, logits.shape, logits.dtype, dev, "dlogits")
    _apart(*logits.shape, logits.element_size(), x, ld, p, pitch)
    return p, pitch


def _rows_apart(T, written, read):
    """Raises where a result [T] (of the addresses ``written``) overlaps another one or an operand [T] (``read``): the
    thread that writes it is not the only one that reads the operand."""
    size = 4 * T
    for k, p in enumerate(written):
        if p:
            for q in written[:k] + read:
                if q and -size < p - q < size:
                    raise ValueError("logp and lse of out must not overlap each other nor another operand")


def _space(workspace, need: int, device: torch.device):
    """The caller's workspace or a new one, its address and size."""
    if workspace is None:
        if need == 0:
            return None, None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
        return workspace, workspace.data_ptr(), need
    return _scratch(workspace, need, device)


def _rows(T, device):
    return torch.empty(T, dtype=_F32, device=device)


@functools.lru_cache(maxsize=1024)   # (of the sizes alone)
def elas_token_loss_workspace_bytes(T: int, V: int, flags: int = 0) -> int:
    """Workspace of elas_token_loss and elas_policy_loss on logits [T, V] (``flags``:
    ELAS_LOGITS_F32 for float32 logits)."""
    return lib().elas_token_loss_workspace_bytes(T, V, flags)


def elas_token_logp_fwd(logits, ids, scale: float = 1.0, out: dict | None = None) -> dict:
    """Log-probabilities of tokens: with z = scale * logits, lse = log sum exp z over
    the vocabulary and logp = z[id] - lse.  logits is [T, V], bf16 or float32, its rows
    contiguous (any pitch and alignment); ids [T] int32 or int64.  A token whose id is
    outside 0 .. V-1 takes no part: its logits are not read, its results are 0.
    Returns dict(logp, lse), float32 [T] (of an ``out`` without lse: logp alone)."""
    T, V, dev, flags, x, ld, ids_p = _logits(logits, ids)
    if out is None:
        out = {"logp": _rows(T, logits.device), "lse": _rows(T, logits.device)}
    logp_p = _arg(_required(out.get("logp"), "out['logp']"), (T,), _F32, dev, "out['logp']")
    lse_p = _opt(out.get("lse"), (T,), _F32, dev, "out['lse']")
    _rows_apart(T, (logp_p, lse_p), ())
    _on(dev, lib().elas_token_logp_fwd, x, ld, ids_p, T, V, scale, flags, logp_p, lse_p)
    return out


def elas_token_logp_bwd(dlogp, logits, ids, lse, scale: float = 1.0, dlse: torch.Tensor | None = None,
                        dlogits: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient of the logits from those of logp and (dlse, None: zero) of lse, at the
    forward's lse: dlogits [T, V] in the logits' type, rows of tokens that take no part
    zeros.  dlogits may be the logits' own tensor."""
    T, V, dev, flags, x, ld, ids_p = _logits(logits, ids)
    if dlogits is None:
        dlogits = torch.empty((T, V), dtype=logits.dtype, device=logits.device)
    d_p, ld_out = _gradient(dlogits, logits, dev, x, ld)
    _on(dev, lib().elas_token_logp_bwd, _arg(dlogp, (T,), _F32, dev, "dlogp"), _opt(dlse, (T,), _F32, dev, "dlse"), x, ld, ids_p,
        _arg(lse, (T,), _F32, dev, "lse"), T, V, scale, flags, d_p, ld_out)
    return dlogits


def elas_token_loss(logits, ids, weight: torch.Tensor | None = None, scale: float = 1.0, reduce: float = 1.0, z_coef: float = 0.0,
                    out: dict | None = None, workspace: torch.Tensor | None = None) -> dict:
    """Cross-entropy of tokens with its gradient, from one pass over the logits:

        loss = reduce * sum_t weight_t (-logp_t + z_coef lse_t^2)

    logits, ids and scale as in elas_token_logp_fwd; weight is float32 [T] or None (1);
    tokens of weight 0 take no part.  Returns dict(stats, logp, lse, dlogits): stats
    float32 [2] holds the loss and its z_coef term.  Of an ``out`` without logp, lse or
    dlogits these are not computed; dlogits may be the logits' own tensor."""
    T, V, dev, flags, x, ld, ids_p = _logits(logits, ids)
    if out is None:
        out = {"stats": _rows(2, logits.device), "logp": _rows(T, logits.device), "lse": _rows(T, logits.device),
               "dlogits": torch.empty((T, V), dtype=logits.dtype, device=logits.device)}
    stats_p = _arg(_required(out.get("stats"), "out['stats']"), (2,), _F32, dev, "out['stats']")
    d_p, ld_out = _gradient(out.get("dlogits"), logits, dev, x, ld)
    row = (T,)
    weight_p = _opt(weight, row, _F32, dev, "weight")
    rows = (_opt(out.get("logp"), row, _F32, dev, "out['logp']"), _opt(out.get("lse"), row, _F32, dev, "out['lse']"))
    _rows_apart(T, rows, (weight_p,))
    workspace, ws_p, ws_n = _space(workspace, elas_token_loss_workspace_bytes(T, V, flags & ELAS_LOGITS_F32), logits.device)
    _on(dev, lib().elas_token_loss, x, ld, ids_p, weight_p, T, V, scale, reduce, z_coef, flags, *rows, d_p, ld_out, stats_p, ws_p, ws_n)
    return out


def elas_policy_loss(logits, ids, advantage, old_logp: torch.Tensor | None = None, ref_logp: torch.Tensor | None = None,
                     weight: torch.Tensor | None = None, scale: float = 1.0, reduce: float = 1.0, clip_low: float = 0.2,
                     clip_high: float = 0.2, kl_coef: float = 0.0, out: dict | None = None, workspace: torch.Tensor | None = None) -> dict:
    """The clipped policy loss with a KL term, and its gradient, from one pass over the
    logits.  With r = exp(logp - old_logp), q = ref_logp - logp and k = exp(q) - q - 1:

        loss = reduce * sum_t weight_t (-min(r A, clamp(r, 1 - clip_low, 1 + clip_high) A) + kl_coef k)

    advantage (A), old_logp, ref_logp and weight are float32 [T]; without old_logp the
    policy is the one that sampled (r = 1, with its gradient), without ref_logp there is
    no KL term.  logits, ids and scale as in elas_token_logp_fwd.  Returns dict(stats,
    logp, dlogits): stats float32 [3] holds the loss, the sum of k and the share of
    tokens that the clamp holds (both times reduce and weight).  Of an ``out`` without logp or dlogits
    these are not computed; dlogits may be the logits' own tensor."""
    T, V, dev, flags, x, ld, ids_p = _logits(logits, ids)
    if out is None:
        out = {"stats": _rows(3, logits.device), "logp": _rows(T, logits.device),
               "dlogits": torch.empty((T, V), dtype=logits.dtype, device=logits.device)}
    stats_p = _arg(_required(out.get("stats"), "out['stats']"), (3,), _F32, dev, "out['stats']")
    d_p, ld_out = _gradient(out.get("dlogits"), logits, dev, x, ld)
    row = (T,)
    rows = (_arg(advantage, row, _F32, dev, "advantage"), _opt(old_logp, row, _F32, dev, "old_logp"),
            _opt(ref_logp, row, _F32, dev, "ref_logp"), _opt(weight, row, _F32, dev, "weight"))
    logp_p = _opt(out.get("logp"), row, _F32, dev, "out['logp']")
    _rows_apart(T, (logp_p,), rows)
    workspace, ws_p, ws_n = _space(workspace, elas_token_loss_workspace_bytes(T, V, flags & ELAS_LOGITS_F32), logits.device)
    _on(dev, lib().elas_policy_loss, x, ld, ids_p, *rows, T, V, scale, reduce, clip_low, clip_high, kl_coef, flags, logp_p, d_p, ld_out, stats_p,
        ws_p, ws_n)
    return out


@functools.lru_cache(maxsize=1024)   # (of the sizes alone)
def elas_preference_loss_workspace_bytes(N: int, pairs: int) -> int:
    return lib().elas_preference_loss_workspace_bytes(N, pairs)


def elas_preference_loss(logp, offsets, ref_logp: torch.Tensor | None = None, beta: float = 0.1, smoothing: float = 0.0,
                         out: dict | None = None, workspace: torch.Tensor | None = None) -> dict:
    """The loss of paired answers by their log-ratios, with its gradient.  Answer s is
    logp[offsets[s]:offsets[s + 1]] (offsets int32 or int64 [2 pairs + 1], rising; chosen
    and rejected in turn).  With z = beta * (the chosen answer's sum of logp - ref_logp,
    less the rejected one's):

        loss = mean over pairs of -(1 - smoothing) log sigmoid(z) - smoothing log sigmoid(-z)

    Returns dict(stats, margin, dlogp): stats float32 [3] holds the loss, the share of
    z > 0 and the mean z; margin [pairs] is z; dlogp is logp's gradient, 0 outside the
    answers.  Of an ``out`` without margin or dlogp these are not computed; dlogp may be logp."""
    if logp.dim() != 1 or offsets.dim() != 1 or offsets.shape[0] % 2 != 1:
        raise ValueError("logp must be 1-D and offsets [2 pairs + 1]")
    N, pairs = logp.shape[0], offsets.shape[0] // 2
    dev = logp.get_device()
    if offsets.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"offsets must be torch.int32 or torch.int64, got {offsets.dtype}")
    flags = ELAS_IDS_I64 if offsets.dtype == torch.int64 else 0
    logp_p = _arg(logp, (N,), _F32, dev, "logp")
    offsets_p = _arg(offsets, (2 * pairs + 1,), offsets.dtype, dev, "offsets")
    if out is None:
        out = {"stats": _rows(3, logp.device), "margin": _rows(pairs, logp.device), "dlogp": torch.empty_like(logp)}
    stats_p = _arg(_required(out.get("stats"), "out['stats']"), (3,), _F32, dev, "out['stats']")
    dlogp_p = _opt(out.get("dlogp"), (N,), _F32, dev, "out['dlogp']")
    for t, name in ((logp_p, "logp"), (None if ref_logp is None else ref_logp.data_ptr(), "ref_logp")):
        if dlogp_p and t and abs(dlogp_p - t) < 4 * N and not (dlogp_p == t and name == "logp"):
            raise ValueError(f"dlogp must be logp itself or overlap nothing of {name}")
    workspace, ws_p, ws_n = _space(workspace, elas_preference_loss_workspace_bytes(N, pairs), logp.device)
    _on(dev, lib().elas_preference_loss, logp_p, _opt(ref_logp, (N,), _F32, dev, "ref_logp"), offsets_p, N, pairs, beta, smoothing, flags,
        _opt(out.get("margin"), (pairs,), _F32, dev, "out['margin']"), dlogp_p, stats_p,
        ws_p, ws_n)
    return out
