"""The measured workloads of the operators around the feed-forward block in a
training step: the norms before and after a block with its gate and residual
scale (``elas_norm_join_*``), the embedding and its gradient (``elas_embed_*``),
and the global gradient norm with clipping (``elas_grad_*``), at the four model
shapes of the paper (Table 6: hidden and intermediate sizes; Table 1: rank).

``listed()`` names the fixed cases and ``draw(rng)`` samples one more from the
same ranges; ``prepare`` makes a case's inputs and buffers on the GPU, ``run``
is one call, ``work`` the bytes and operations it cannot do without, ``exact``
the same outputs in 64-bit arithmetic.  Where ``own`` is false ``run`` computes
the plain form instead, in elementary torch operations.
"""
import math

import torch

own = False

# name -> (d, d_ff, r, layers)
MODELS = {
    "60m": (512, 1376, 128, 8),
    "130m": (768, 2048, 256, 12),
    "350m": (1024, 2736, 256, 24),
    "1b": (2048, 5461, 512, 32),
}
VOCAB = 32000
EPS = 1e-6

# Tokens each kind of call is made with: a generated token or a batch of
# prompts (forward), one GPU's share of a training batch (backward).
TOKENS = {
    "join_fwd": (1, 65536),
    "join_bwd": (256, 65536),
    "embed_fwd": (1, 65536),
    "embed_bwd": (256, 65536),
}


def _case(name, kind, model, **more):
    return dict(name=name, kind=kind, model=model, **more)


def listed():
    return [
        # serving, one step of 16 sequences between two blocks: latency only
        _case("join_fwd_1b_t16", "join_fwd", "1b", tokens=16, post=True, gate="shared", pre=True, res="bf16"),
        # a prompt of 2000 tokens (no multiple of a tile) with a gate per token
        _case("join_fwd_350m_t2000", "join_fwd", "350m", tokens=2000, post=True, gate="token", pre=True, res="bf16"),
        # the largest training batch, the residual stream kept in float32
        _case("join_fwd_1b_t65536", "join_fwd", "1b", tokens=65536, post=True, gate="shared", pre=True, res="f32"),
        # the plain pre-norm block (residual sum and norm) on one short batch
        _case("join_bwd_60m_t2048", "join_bwd", "60m", tokens=2048, post=False, gate="none", pre=True, res="bf16"),
        # an ordinary micro-batch, ragged, gate per token
        _case("join_bwd_350m_t16381", "join_bwd", "350m", tokens=16381, post=True, gate="token", pre=True, res="f32"),
        # the largest training batch
        _case("join_bwd_1b_t65536", "join_bwd", "1b", tokens=65536, post=True, gate="shared", pre=True, res="bf16"),
        # ids of a ragged batch with padding
        _case("embed_fwd_130m_t8191", "embed_fwd", "130m", tokens=8191, ids="i64", padding=0.25, res="bf16"),
        # a short micro-batch added to the gradient of the ones before it
        _case("embed_bwd_60m_t2048", "embed_bwd", "60m", tokens=2048, ids="i64", padding=0.0, res="bf16", accumulate=True),
        # the largest training batch: frequent tokens come thousands of times
        _case("embed_bwd_1b_t65536", "embed_bwd", "1b", tokens=65536, ids="i32", padding=0.0, res="bf16", accumulate=False),
        # the norm alone, for logging: types mixed, lengths odd, no alignment
        _case("norm_130m_ragged", "norm", "130m", types="mixed", odd=True),
        # all gradients of the smallest and of the largest model
        _case("clip_60m", "clip", "60m", types="f32", odd=False, clips=True),
        _case("clip_1b", "clip", "1b", types="f32", odd=False, clips=True),
    ]


def draw(rng):
    kind = rng.choice(["join_fwd", "join_fwd", "join_bwd", "join_bwd", "embed_fwd", "embed_bwd", "embed_bwd", "norm", "clip"])
    case = {"kind": kind, "model": rng.choice(sorted(MODELS))}
    if kind in TOKENS:
        lo, hi = TOKENS[kind]
        case["tokens"] = min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))
        case["res"] = rng.choice(["bf16", "f32"])
    if kind.startswith("join"):
        case["post"] = rng.random() < 0.6
        case["gate"] = rng.choice(["none", "shared", "token"])
        case["pre"] = rng.random() < 0.85
    elif kind.startswith("embed"):
        case["ids"] = rng.choice(["i32", "i64"])
        case["padding"] = round(rng.choice([0.0, rng.uniform(0.0, 0.5)]), 3)
        if kind == "embed_bwd":
            case["accumulate"] = rng.random() < 0.5
    else:
        case["types"] = rng.choice(["f32", "bf16", "mixed"])
        case["odd"] = rng.random() < 0.5
        case["layers"] = rng.randint(1, MODELS[case["model"]][3])
        if kind == "clip":
            case["clips"] = rng.random() < 0.8
    return case


# ---- inputs ------------------------------------------------------------------


def _randn(gen, shape, sigma=1.0, dtype=torch.bfloat16, mean=0.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(sigma).add_(mean).to(dtype)


def _join_inputs(case, seed):
    """The residual stream and a block's output about N(0, 1) and N(0, 1/4),
    gains near 1, gradients of a mean over tokens."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    d, _, _, layers = MODELS[case["model"]]
    t = case["tokens"]
    res = torch.float32 if case["res"] == "f32" else torch.bfloat16
    i = {"h": _randn(gen, (t, d), dtype=res), "b": _randn(gen, (t, d), 0.5), "gate": None, "w_post": None, "w_pre": None,
         "res_scale": 1.0, "block_scale": (2 * layers) ** -0.5}
    if case["gate"] != "none":
        i["gate"] = _randn(gen, (t, d) if case["gate"] == "token" else (d,), 0.25, mean=0.75)
    if case["post"]:
        i["w_post"] = _randn(gen, (d,), 0.1, mean=1.0)
    if case["pre"]:
        i["w_pre"] = _randn(gen, (d,), 0.1, mean=1.0)
    if case["kind"] == "join_bwd":
        i["dh"] = _randn(gen, (t, d), 0.02, dtype=res)
        i["dn"] = _randn(gen, (t, d), 0.02) if case["pre"] else None
    return i


def _embed_inputs(case, seed):
    """Ids that fall off like words do (about the inverse of their rank), a
    share of them padding (-1)."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    d, _, _, _ = MODELS[case["model"]]
    t = case["tokens"]
    rank = torch.arange(VOCAB, device="cuda", dtype=torch.float64)
    cdf = torch.cumsum(1.0 / (rank + 2.7), 0)
    u = torch.rand(t, generator=gen, device="cuda", dtype=torch.float64) * cdf[-1]
    ids = torch.searchsorted(cdf, u).clamp_max_(VOCAB - 1)
    if case["padding"]:
        ids[torch.rand(t, generator=gen, device="cuda") < case["padding"]] = -1
    res = torch.float32 if case["res"] == "f32" else torch.bfloat16
    i = {"ids": ids.to(torch.int32) if case["ids"] == "i32" else ids, "scale": d ** 0.5, "res": res}
    if case["kind"] == "embed_fwd":
        i["table"] = _randn(gen, (VOCAB, d), d ** -0.5)
    else:
        i["dx"] = _randn(gen, (t, d), 0.02, dtype=res)
        if case["accumulate"]:
            i["dtable"] = _randn(gen, (VOCAB, d), 0.02, dtype=torch.float32)
    return i


def _grad_lengths(case):
    """Values of each gradient: per layer the four factors and two norm gains
    (and, where ``odd``, a learned scale of one value), then the final norm."""
    d, f, r, layers = MODELS[case["model"]]
    if not case["odd"]:
        f = -(-f // 8) * 8
    layer = [d * r, r * f, f * r, r * d, d, d] + ([1] if case["odd"] else [])
    return layer * case.get("layers", layers) + [d]


def _is_bf16(case, k):
    return case["types"] == "bf16" or (case["types"] == "mixed" and k % 3 == 1)


def _grad_flat(case, seed):
    """The gradients as programs keep them: one flat buffer for each type."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lengths = _grad_lengths(case)
    flat = {}
    for key, dtype in (("bf16", torch.bfloat16), ("f32", torch.float32)):
        total = sum(n for k, n in enumerate(lengths) if _is_bf16(case, k) == (key == "bf16"))
        if total:
            flat[key] = torch.empty(total, dtype=dtype, device="cuda")
            for piece in flat[key].split(1 << 26):
                piece.copy_(torch.randn(piece.shape, generator=gen, device="cuda").mul_(1e-2))
    return flat


def _grad_views(case, flat):
    at = dict.fromkeys(flat, 0)
    views = []
    for k, n in enumerate(_grad_lengths(case)):
        key = "bf16" if _is_bf16(case, k) else "f32"
        views.append(flat[key][at[key]:at[key] + n])
        at[key] += n
    return views


def _max_norm(case):
    """Well under the gradients' norm where the case clips, well over it where not."""
    return (0.1 if case["clips"] else 10.0) * 1e-2 * sum(_grad_lengths(case)) ** 0.5


def prepare(case, seed):
    kind = case["kind"]
    if kind.startswith("join"):
        s = {"case": case, **_join_inputs(case, seed)}
        t, d = s["h"].shape
        if kind == "join_fwd":
            # the buffers a program keeps from step to step
            s["out"] = {"h": torch.empty_like(s["h"]),
                        "n": torch.empty((t, d), dtype=torch.bfloat16, device="cuda") if case["pre"] else None}
        else:
            per_token, shared = case["gate"] == "token", case["gate"] == "shared"
            sums = {"dgate": shared, "dw_post": case["post"], "dw_pre": case["pre"]}
            s["out"] = {k: torch.empty(d, dtype=torch.float32, device="cuda") if there else None for k, there in sums.items()}
            s["out"]["dh"], s["out"]["db"] = torch.empty_like(s["dh"]), torch.empty_like(s["b"])
            if per_token:
                s["out"]["dgate"] = torch.empty_like(s["gate"])
        return s
    if kind.startswith("embed"):
        s = {"case": case, **_embed_inputs(case, seed)}
        if kind == "embed_bwd" and not case["accumulate"]:
            s["dtable"] = torch.empty((VOCAB, s["dx"].shape[1]), dtype=torch.float32, device="cuda")
        return s
    flat = _grad_flat(case, seed)
    s = {"case": case, "grads": _grad_views(case, flat)}
    if kind == "clip":
        s["flat"] = {k: torch.empty_like(v) for k, v in flat.items()}
        s["clipped"] = _grad_views(case, s["flat"])
        s["max_norm"] = _max_norm(case)
    if own:
        # the lists of tensors, made once as an optimizer makes its parameter groups
        import paper_2605_03667_amd as elas
        s["grads"] = elas.ElasTensors(s["grads"])
        if kind == "clip":
            s["clipped"] = elas.ElasTensors(s["clipped"])
    return s


# ---- the framework's calls -----------------------------------------------------


def _run_own(s):
    import paper_2605_03667_amd as elas

    kind = s["case"]["kind"]
    if kind == "join_fwd":
        o = elas.elas_norm_join_fwd(s["h"], s["b"], s["gate"], s["w_post"], s["w_pre"], res_scale=s["res_scale"],
                                    block_scale=s["block_scale"], eps=EPS, out=s["out"])
        return {k: o[k] for k in ("h", "n") if o[k] is not None}
    if kind == "join_bwd":
        g = elas.elas_norm_join_bwd(s["dh"], s["dn"], s["h"], s["b"], s["gate"], s["w_post"], s["w_pre"],
                                    res_scale=s["res_scale"], block_scale=s["block_scale"], eps=EPS, grads=s["out"])
        return {k: v for k, v in g.items() if v is not None}
    if kind == "embed_fwd":
        return {"x": elas.elas_embed_fwd(s["ids"], s["table"], s["scale"], dtype=s["res"])}
    if kind == "embed_bwd":
        return {"dtable": elas.elas_embed_bwd(s["ids"], s["dx"], VOCAB, s["scale"], dtable=s["dtable"],
                                              accumulate=s["case"]["accumulate"])}
    if kind == "norm":
        return {"norm": elas.elas_grad_norm(s["grads"])}
    return {"stats": elas.elas_grad_clip(s["grads"], s["max_norm"], out=s["clipped"]), **s["flat"]}


# ---- the plain form --------------------------------------------------------------


def _rms(x):
    return torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)


def _plain_join_fwd(s):
    u = s["b"].float()
    if s["w_post"] is not None:
        u = u * _rms(u) * s["w_post"].float()
    if s["gate"] is not None:
        u = u * s["gate"].float()
    h = s["res_scale"] * s["h"].float() + s["block_scale"] * u
    out = {"h": h.to(s["h"].dtype)}
    if s["w_pre"] is not None:
        out["n"] = (h * _rms(h) * s["w_pre"].float()).to(torch.bfloat16)
    return out


def _plain_join_bwd(s):
    g = s["dh"].float()
    out = {}
    if s["w_pre"] is not None:
        h, dn = s["h"].float(), s["dn"].float()
        sig = _rms(h)
        xh = h * sig
        q = dn * s["w_pre"].float()
        g = g + sig * (q - xh * (q * xh).mean(1, keepdim=True))
        out["dw_pre"] = (dn * xh).sum(0)
    out["dh"] = (s["res_scale"] * g).to(s["dh"].dtype)
    b = s["b"].float()
    rho = _rms(b) if s["w_post"] is not None else None
    bh = b * rho if rho is not None else b
    du = s["block_scale"] * g
    if s["gate"] is not None:
        dgate = du * (bh * s["w_post"].float() if rho is not None else bh)
        out["dgate"] = dgate.sum(0) if s["gate"].dim() == 1 else dgate.to(torch.bfloat16)
        du = du * s["gate"].float()
    if rho is not None:
        out["dw_post"] = (du * bh).sum(0)
        p = du * s["w_post"].float()
        du = rho * (p - bh * (p * bh).mean(1, keepdim=True))
    out["db"] = du.to(torch.bfloat16)
    return out


def _plain_embed_fwd(s):
    ids = s["ids"].long()
    inside = (ids >= 0) & (ids < VOCAB)
    rows = s["table"][torch.where(inside, ids, 0)].float() * s["scale"]
    return {"x": torch.where(inside[:, None], rows, 0.0).to(s["res"])}


def _plain_embed_bwd(s):
    ids = s["ids"].long()
    inside = (ids >= 0) & (ids < VOCAB)
    rows = torch.where(inside[:, None], s["dx"].float() * s["scale"], 0.0)
    if not s["case"]["accumulate"]:
        s["dtable"].zero_()
    return {"dtable": s["dtable"].index_add_(0, torch.where(inside, ids, 0), rows)}


def _plain_norm(grads):
    return torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()


def _plain_clip(s):
    norm = _plain_norm(s["grads"])
    factor = (s["max_norm"] / norm).clamp_max(1.0)
    [o.copy_(g.float() * factor) for g, o in zip(s["grads"], s["clipped"])]
    return {"stats": torch.stack([norm, factor]), **s["flat"]}


def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    if kind == "join_fwd":
        return _plain_join_fwd(s)
    if kind == "join_bwd":
        return _plain_join_bwd(s)
    if kind == "embed_fwd":
        return _plain_embed_fwd(s)
    if kind == "embed_bwd":
        return _plain_embed_bwd(s)
    if kind == "norm":
        return {"norm": _plain_norm(s["grads"]).reshape(1)}
    return _plain_clip(s)


# ---- what a call cannot do without -------------------------------------------------


def work(case):
    """Inputs read once, outputs written once."""
    kind = case["kind"]
    if kind in ("norm", "clip"):
        lengths = _grad_lengths(case)
        size = sum(n * (2 if _is_bf16(case, k) else 4) for k, n in enumerate(lengths))
        return {"bytes": size * (2 if kind == "clip" else 1) + 8, "flops": (3 if kind == "clip" else 2) * sum(lengths)}
    d = MODELS[case["model"]][0]
    t = case["tokens"]
    res = 4 if case["res"] == "f32" else 2
    if kind.startswith("embed"):
        id_bytes = t * (4 if case["ids"] == "i32" else 8)
        rows = t * (1 - case["padding"])                 # tokens that have a row
        # distinct rows among them: the expected number under the inputs' distribution
        total = sum(1.0 / (k + 2.7) for k in range(VOCAB))
        distinct = sum(1.0 - (1.0 - 1.0 / ((k + 2.7) * total)) ** rows for k in range(VOCAB))
        if kind == "embed_fwd":
            return {"bytes": id_bytes + 2 * distinct * d + res * t * d, "flops": rows * d}
        table = 8 * distinct * d if case["accumulate"] else 4 * VOCAB * d
        return {"bytes": id_bytes + res * rows * d + table, "flops": rows * d}
    gate = {"none": 0, "shared": 0, "token": 2}[case["gate"]]
    if kind == "join_fwd":
        per = 2 * res + 2 + gate + (2 if case["pre"] else 0)
        return {"bytes": per * t * d + 2 * d * (case["post"] + case["pre"] + (case["gate"] == "shared")), "flops": 12 * t * d}
    per = 2 * res + 4 + 2 * gate + ((2 + res) if case["pre"] else 0)
    sums = case["post"] + case["pre"] + (case["gate"] == "shared")
    return {"bytes": per * t * d + 6 * d * sums, "flops": 25 * t * d}


# ---- 64 bits ------------------------------------------------------------------------


def exact(case, seed):
    kind = case["kind"]
    if kind in ("norm", "clip"):
        flat = _grad_flat(case, seed)
        square = sum(float((p.double() ** 2).sum()) for v in flat.values() for p in v.split(1 << 26))
        norm = math.sqrt(square)
        if kind == "norm":
            return {"norm": torch.tensor([norm], dtype=torch.float64)}
        factor = min(1.0, _max_norm(case) / norm)
        return {"stats": torch.tensor([norm, factor], dtype=torch.float64), **{k: v.double() * factor for k, v in flat.items()}}
    if kind.startswith("embed"):
        i = _embed_inputs(case, seed)
        ids = i["ids"].long()
        if kind == "embed_fwd":
            x = i["table"].double()[ids] * i["scale"]     # -1 takes the last row, cleared below
            x[ids < 0] = 0
            return {"x": x}
        # sums of runs of equal ids as differences of running sums
        order = torch.argsort(ids, stable=True)
        order = order[ids[order] >= 0]
        v, count = torch.unique_consecutive(ids[order], return_counts=True)
        ends = torch.cumsum(count, 0)
        out = i["dtable"].double() if case["accumulate"] else torch.zeros((VOCAB, i["dx"].shape[1]), dtype=torch.float64, device="cuda")
        if len(v):
            run_sum = torch.cumsum(i["dx"][order].double(), 0)[ends - 1]
            out[v] += i["scale"] * torch.diff(run_sum, dim=0, prepend=torch.zeros_like(run_sum[:1]))
        return {"dtable": out}
    i = {k: v.double() if isinstance(v, torch.Tensor) else v for k, v in _join_inputs(case, seed).items()}
    h, b, d = i["h"], i["b"], i["h"].shape[1]
    gate = 1.0 if i["gate"] is None else i["gate"]
    gain = 1.0 if i["w_post"] is None else i["w_post"]
    rho = 1.0 if i["w_post"] is None else 1.0 / ((b ** 2).sum(1, keepdim=True) / d + EPS).sqrt()
    if kind == "join_fwd":
        h = i["res_scale"] * h + i["block_scale"] * gate * (b * rho * gain)
        out = {"h": h}
        if case["pre"]:
            out["n"] = h * i["w_pre"] / ((h ** 2).sum(1, keepdim=True) / d + EPS).sqrt()
        return out
    total = i["dh"]
    out = {}
    if case["pre"]:
        # n = w h s^(-1/2) with s = |h|^2 / d + eps
        s = (h ** 2).sum(1, keepdim=True) / d + EPS
        out["dw_pre"] = (i["dn"] * h / s.sqrt()).sum(0)
        q = i["dn"] * i["w_pre"]
        total = total + q / s.sqrt() - h * (q * h).sum(1, keepdim=True) / (d * s ** 1.5)
    out["dh"] = i["res_scale"] * total
    if i["gate"] is not None:
        dgate = i["block_scale"] * total * gain * rho * b
        out["dgate"] = dgate if case["gate"] == "token" else dgate.sum(0)
    p = i["block_scale"] * total * gate
    if i["w_post"] is not None:
        out["dw_post"] = (p * rho * b).sum(0)
        p = p * gain
        p = rho * p - rho ** 3 * b * (p * b).sum(1, keepdim=True) / d
    out["db"] = p
    return out
