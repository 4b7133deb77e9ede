"""The measured workloads of the operators that begin and end the backward half
of a training step: the log-probabilities of tokens from logits with their
gradient (``elas_token_logp_*``), the losses on them (``elas_token_loss``,
``elas_policy_loss``, ``elas_preference_loss``), and the AdamW step over many
tensors with states in 32 or 8 bits (``elas_adamw_step``), at the vocabulary and
the four model shapes of the paper (Table 6: hidden and intermediate sizes;
Table 1: rank).

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
BLOCK = 256                       # values of a state in 8 bits that share a scale
SCORED = 1 << 30                  # most logits of a drawn case

# Hyper-parameters of the update: the usual ones of language models.
RATE, BETA1, BETA2, EPS, DECAY = 3e-4, 0.9, 0.95, 1e-8, 0.1


def _case(name, kind, **more):
    return dict(name=name, kind=kind, **more)


def _logits(tokens, vocab, dtype="bf16", padding=0.0, pitch=0, banned=0.0, scale=1.0, ids="i64"):
    """pitch: logits of a row behind the vocabulary (a padded head), banned: share
    of the vocabulary whose logits are -inf, scale: 1 / temperature."""
    return dict(tokens=tokens, vocab=vocab, dtype=dtype, padding=padding, pitch=pitch, banned=banned, scale=scale, ids=ids)


def listed():
    return [
        # serving: the tokens just sampled for 16 sequences, with a temperature; latency only
        _case("logp_fwd_t16", "logp_fwd", **_logits(16, VOCAB, scale=1.25)),
        # scoring of prompts with the reference model: ragged, float32 logits, an odd vocabulary
        _case("logp_fwd_t4093_odd", "logp_fwd", **_logits(4093, 32003, dtype="f32", padding=0.25)),
        # gradient of log-probabilities that a loss of the program's own was computed from
        _case("logp_bwd_t8192", "logp_bwd", **_logits(8192, VOCAB)),
        # pre-training, a short micro-batch of the smallest vocabulary
        _case("token_loss_v1000_t2048", "token_loss", **_logits(2048, 1000, ids="i32"), weights=False),
        # pre-training: a micro-batch with padding, the head padded to a multiple of 128 rows
        _case("token_loss_t16381", "token_loss", **_logits(16381, VOCAB, padding=0.125, pitch=128), weights=True),
        # policy optimisation: one micro-batch, the prompts masked, some tokens banned
        _case("policy_t2000", "policy", **_logits(2000, VOCAB, dtype="f32", padding=0.25, banned=0.01), kl=0.05, old=True),
        # policy optimisation: the largest batch
        _case("policy_t65536", "policy", **_logits(65536, VOCAB), kl=0.02, old=True),
        # preference optimisation: a few pairs of short answers, and a large batch of long ones
        _case("preference_p8", "preference", pairs=8, length=100, smoothing=0.0, ref=True, offsets="i32"),
        _case("preference_p2048", "preference", pairs=2048, length=1000, smoothing=0.1, ref=True, offsets="i64"),
        # the update of the smallest model, of a mixed one with odd lengths, and of the largest with states in 8 bits
        _case("adamw_60m", "adamw", model="60m", bits=32, params="f32+copy", grads="f32", odd=False, clip=True),
        _case("adamw_350m_odd", "adamw", model="350m", bits=32, params="f32", grads="bf16", odd=True, clip=False),
        _case("adamw8_1b", "adamw", model="1b", bits=8, params="f32+copy", grads="f32", odd=False, clip=True),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["logp_fwd", "logp_bwd", "token_loss", "token_loss", "policy", "policy", "preference", "adamw", "adamw", "adamw"])
    case = {"kind": kind}
    if kind == "preference":
        case.update(pairs=_log_uniform(rng, 1, 2048), length=_log_uniform(rng, 1, 1000), smoothing=rng.choice([0.0, 0.1]),
                    ref=rng.random() < 0.8, offsets=rng.choice(["i32", "i64"]))
    elif kind == "adamw":
        model = rng.choice(sorted(MODELS))
        case.update(model=model, layers=rng.randint(1, MODELS[model][3]), bits=rng.choice([8, 32]), params=rng.choice(["f32", "f32+copy", "bf16"]),
                    grads=rng.choice(["f32", "bf16"]), odd=rng.random() < 0.5, clip=rng.random() < 0.5)
    else:
        vocab = rng.choice([VOCAB, _log_uniform(rng, 1000, 131072)])
        case.update(_logits(min(_log_uniform(rng, 1, 65536), SCORED // vocab), vocab, dtype=rng.choice(["bf16", "f32"]),
                            padding=round(rng.choice([0.0, rng.uniform(0.0, 0.5)]), 3), pitch=rng.choice([0, 0, rng.randint(1, 128)]),
                            banned=rng.choice([0.0, 0.01]), scale=rng.choice([1.0, 1.25]), ids=rng.choice(["i32", "i64"])))
        if kind == "token_loss":
            case["weights"] = rng.random() < 0.5
        elif kind == "policy":
            case.update(kl=rng.choice([0.0, 0.05]), old=rng.random() < 0.7)
    return case


# ---- inputs: logits ------------------------------------------------------------


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _log_probabilities(logits, ids, scale):
    """In 64 bits, a few rows at a time; 0 where an id is outside the vocabulary."""
    t, v = logits.shape
    out = torch.zeros(t, dtype=torch.float64, device=logits.device)
    step = max(1, (1 << 27) // v)
    for a in range(0, t, step):
        z = logits[a:a + step].double() * scale
        i = ids[a:a + step].long()
        there = (i >= 0) & (i < v)
        label = z.gather(1, torch.where(there, i, 0)[:, None])[:, 0]
        out[a:a + step] = torch.where(there, label - torch.logsumexp(z, 1), 0.0)
    return out


def _logit_inputs(case, seed):
    """Logits about N(0, 4) with the next token's raised, so that its probability
    lies between 1e-6 and nearly 1; prompts and padding have the id -1."""
    gen = _generator(seed)
    t, v = case["tokens"], case["vocab"]
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    full = torch.randn((t, v + case["pitch"]), generator=gen, device="cuda", dtype=dtype).mul_(2.0)
    logits = full[:, :v]
    if case["banned"]:
        logits.masked_fill_((torch.rand(v, generator=gen, device="cuda") < case["banned"])[None], -math.inf)
    ids = torch.randint(0, v, (t, 1), generator=gen, device="cuda")
    raised = torch.randn((t, 1), generator=gen, device="cuda") * 3.0 + 0.8 * math.log(v)
    logits.scatter_(1, ids, raised.to(dtype))
    ids = ids[:, 0]
    if case["padding"]:
        ids[torch.rand(t, generator=gen, device="cuda") < case["padding"]] = -1
    i = {"logits": logits, "ids": ids.to(torch.int32) if case["ids"] == "i32" else ids, "scale": case["scale"], "reduce": 1.0 / t}

    def rand(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    kind = case["kind"]
    if kind == "logp_bwd":
        i["dlogp"], i["dlse"] = rand(t) / t, 0.1 * rand(t) / t
        lse = torch.cat([torch.logsumexp(p.double() * case["scale"], 1) for p in logits.split(max(1, (1 << 27) // v))])
        i["lse"] = lse.float()
    elif kind == "token_loss":
        # a weight for each token (by its document), some of them 0
        i["weight"] = rand(t).abs_().sub_(0.2).clamp_min_(0.0) if case["weights"] else None
        i["z_coef"] = 1e-4
    elif kind == "policy":
        # log-probabilities of the policy that sampled the tokens and of the reference model
        logp = _log_probabilities(logits, i["ids"], case["scale"]).float()
        i["kl"], i["low"], i["high"] = case["kl"], 0.2, 0.28
        # (no ratio so near a border of the clipping that rounding would decide on which side it is)
        change = 0.15 * rand(t)
        for border in (-math.log(1.0 - i["low"]), -math.log(1.0 + i["high"])):
            change = torch.where((change - border).abs() < 1e-4, change + 3e-4, change)
        i["old"] = logp + change if case["old"] else None
        i["ref"] = logp + 0.3 * rand(t) if case["kl"] else None
        i["advantage"] = rand(t)
        i["weight"] = 0.5 + torch.rand(t, generator=gen, device="cuda")
    return i


def _logit_outputs(case):
    """The buffers that a program keeps from step to step."""
    t, v = case["tokens"], case["vocab"]
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    out = {"logp": torch.empty(t, device="cuda")}
    if case["kind"] in ("logp_fwd", "token_loss"):
        out["lse"] = torch.empty(t, device="cuda")
    if case["kind"] != "logp_fwd":
        out["dlogits"] = torch.empty((t, v + case["pitch"]), dtype=dtype, device="cuda")[:, :v]
    if case["kind"] in ("token_loss", "policy"):
        out["stats"] = torch.empty(2 if case["kind"] == "token_loss" else 3, device="cuda")
    return out


# ---- inputs: pairs ----------------------------------------------------------------


def _pair_inputs(case, seed):
    """Log-probabilities of answers of 1 to 2 * length tokens, chosen and rejected in
    turn, and what the reference model gives them.  The tokens in all are the same
    for every seed: half the answers are as long as the other half leaves."""
    gen = _generator(seed)
    half = torch.randint(1, 2 * case["length"] + 1, (case["pairs"],), generator=gen, device="cuda")
    order = torch.randperm(2 * case["pairs"], generator=gen, device="cuda")
    lengths = torch.cat([half, 2 * case["length"] + 1 - half])[order]
    offsets = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
    n = int(offsets[-1])
    logp = -torch.rand(n, generator=gen, device="cuda").mul_(0.98).add_(0.01).log_().square_()
    ref = logp + torch.randn(n, generator=gen, device="cuda") * 0.3 if case["ref"] else None
    return {"logp": logp, "ref": ref, "offsets": offsets.to(torch.int32) if case["offsets"] == "i32" else offsets,
            "beta": 0.1, "smoothing": case["smoothing"]}


# ---- inputs: the update ------------------------------------------------------------


def _lengths(case):
    """Values of each tensor and its weight decay: per layer the four factors and
    two norm gains (and, where ``odd``, a learned scale of one value and an odd
    width), then the final norm."""
    d, f, r, layers = MODELS[case["model"]]
    if not case["odd"]:
        f = -(-f // 8) * 8
    else:
        f -= 1 - f % 2
    layer = [(d * r, DECAY), (r * f, DECAY), (f * r, DECAY), (r * d, DECAY), (d, 0.0), (d, 0.0)] + ([(1, 0.0)] if case["odd"] else [])
    return layer * case.get("layers", layers) + [(d, 0.0)]


def _starts(case):
    """First value of each tensor in flat buffers in which each begins a block, and the buffers' length."""
    at, starts = 0, []
    for n, _ in _lengths(case):
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    return starts, at


def _tensor_of_block(case):
    """Per block: its tensor's number, decay and first block."""
    lengths, (starts, _) = _lengths(case), _starts(case)
    blocks = torch.tensor([-(-n // BLOCK) for n, _ in lengths])
    number = torch.repeat_interleave(torch.arange(len(lengths)), blocks)
    return (number.cuda(), torch.tensor([w for _, w in lengths], dtype=torch.float64)[number].cuda(),
            (torch.tensor(starts) // BLOCK)[number].cuda())


def _views(case, flat, shift):
    starts, _ = _starts(case)
    return [flat[shift + a:shift + a + n] for a, (n, _) in zip(starts, _lengths(case))]


def _nearest_codes(x, mantissa, top):
    """Codes and scales of states to begin with (``x`` [blocks, 256], not negative): the nearest."""
    scale = x.amax(1, keepdim=True) / top
    y = x / torch.where(scale > 0, scale, 1.0)
    step = torch.exp2((torch.floor(torch.log2(y.clamp_min(1.0))) - mantissa).clamp_min(0.0))
    y = torch.round(y / step) * step
    e = (torch.floor(torch.log2(y.clamp_min(1.0))) - mantissa + 1).clamp_min(0.0)
    code = e * 2 ** mantissa + y / torch.exp2((e - 1).clamp_min(0.0)) - torch.where(e > 0, 2.0 ** mantissa, 0.0)
    return code.clamp_(0, 2 ** (mantissa + 4) - 1).to(torch.uint8), scale[:, 0].float()


def _update_inputs(case, seed):
    """Weights, gradients and moments in flat buffers (what lies between the tensors
    is 0).  The gradients' sizes differ from block to block; one block in 16 has
    none (an unused row), its moments only fade."""
    gen = _generator(seed)
    starts, total = _starts(case)
    shift = 1 if case["odd"] else 0
    used = torch.zeros(total, dtype=torch.bool, device="cuda")
    for v in _views(case, used, 0):
        v.fill_(True)
    used = used.view(-1, BLOCK)
    size = torch.exp(torch.randn((len(used), 1), generator=gen, device="cuda")) * 1e-3

    def normal():
        return torch.randn(used.shape, generator=gen, device="cuda") * used

    def placed(x, dtype):
        flat = torch.zeros(total + 8, dtype=dtype, device="cuda")
        flat[shift:shift + total] = x.reshape(-1)
        return flat

    grad = normal() * size * (torch.rand((len(used), 1), generator=gen, device="cuda") > 1 / 16)
    m, v = normal() * size * 0.3, (0.3 + normal().square()) * used * size * size
    i = {"p": placed(normal() * 0.02, torch.bfloat16 if case["params"] == "bf16" else torch.float32),
         "g": placed(grad, torch.bfloat16 if case["grads"] == "bf16" else torch.float32),
         "copy": placed(normal(), torch.bfloat16) if case["params"] == "f32+copy" else None,
         "step": torch.full((1,), 100, dtype=torch.int64, device="cuda"),
         "norm": None, "max_norm": 1.0}
    if case["clip"]:
        i["norm"] = grad.double().square().sum().sqrt().float().reshape(1)
        i["max_norm"] = 0.4 * 1e-3 * sum(n for n, _ in _lengths(case)) ** 0.5
    if case["bits"] == 8:
        code, i["m_scale"] = _nearest_codes(m.abs(), 3, 245760.0)
        i["m"] = (code | (m < 0).to(torch.uint8) << 7).reshape(-1)
        code, i["v_scale"] = _nearest_codes(v, 4, 507904.0)
        i["v"] = code.reshape(-1)
    else:
        i["m"], i["v"] = m.reshape(-1), v.reshape(-1)
    return i


def prepare(case, seed):
    kind = case["kind"]
    if kind == "preference":
        s = {"case": case, **_pair_inputs(case, seed)}
        s["out"] = {"stats": torch.empty(3, device="cuda"), "margin": torch.empty(case["pairs"], device="cuda"),
                    "dlogp": torch.empty_like(s["logp"])}
        return s
    if kind != "adamw":
        return {"case": case, **_logit_inputs(case, seed), "out": _logit_outputs(case)}
    s = {"case": case, **_update_inputs(case, seed)}
    s["number"], s["decay"], s["first"] = _tensor_of_block(case)
    if case["bits"] == 8:
        s["values"] = [torch.empty(len(s["m"]), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    if own:
        # the optimizer's state, made once
        import paper_2605_03667_amd as elas
        shift = 1 if case["odd"] else 0
        s["opt"] = elas.ElasAdamW(_views(case, s["p"], shift), copies=None if s["copy"] is None else _views(case, s["copy"], shift),
                                  decay=[w for _, w in _lengths(case)], bits=case["bits"])
        s["grads"] = elas.ElasTensors(_views(case, s["g"], shift))
        for k in ("m", "v", "step") + (("m_scale", "v_scale") if case["bits"] == 8 else ()):
            getattr(s["opt"], k).copy_(s[k])
    return s


# ---- the framework's calls -----------------------------------------------------


def _run_own(s):
    import paper_2605_03667_amd as elas

    case = s["case"]
    kind = case["kind"]
    if kind == "logp_fwd":
        return elas.elas_token_logp_fwd(s["logits"], s["ids"], scale=s["scale"], out=s["out"])
    if kind == "logp_bwd":
        return {"dlogits": elas.elas_token_logp_bwd(s["dlogp"], s["logits"], s["ids"], s["lse"], scale=s["scale"], dlse=s["dlse"],
                                                    dlogits=s["out"]["dlogits"])}
    if kind == "token_loss":
        return elas.elas_token_loss(s["logits"], s["ids"], weight=s["weight"], scale=s["scale"], reduce=s["reduce"], z_coef=s["z_coef"],
                                    out=s["out"])
    if kind == "policy":
        return elas.elas_policy_loss(s["logits"], s["ids"], s["advantage"], old_logp=s["old"], ref_logp=s["ref"], weight=s["weight"],
                                     scale=s["scale"], reduce=s["reduce"], clip_low=s["low"], clip_high=s["high"], kl_coef=s["kl"],
                                     out=s["out"])
    if kind == "preference":
        return elas.elas_preference_loss(s["logp"], s["offsets"], ref_logp=s["ref"], beta=s["beta"], smoothing=s["smoothing"], out=s["out"])
    opt = s["opt"]
    elas.elas_adamw_step(opt, s["grads"], RATE, beta1=BETA1, beta2=BETA2, eps=EPS, norm=s["norm"], max_norm=s["max_norm"])
    out = {"p": s["p"], "step": opt.step, "m": opt.m, "v": opt.v}
    if case["bits"] == 8:
        out["m"] = elas.elas_adam8_values(opt.m, opt.m_scale, out=s["values"][0])
        out["v"] = elas.elas_adam8_values(opt.v, opt.v_scale, second=True, out=s["values"][1])
    if s["copy"] is not None:
        out["copy"] = s["copy"]
    return out


# ---- the plain form --------------------------------------------------------------


def _plain_rows(s):
    """exp(z - max) with its sum in 64 bits, the label's place, log-probability and lse."""
    logits, ids = s["logits"], s["ids"].long()
    keep = (ids >= 0) & (ids < logits.shape[1])
    if s.get("weight") is not None:
        keep = keep & (s["weight"] != 0)
    label = torch.where(keep, ids, 0)[:, None]
    z = logits.float() * s["scale"]
    top = z.amax(1, keepdim=True)
    z_label = z.gather(1, label).double()
    e = z.sub_(top).exp_()
    total = e.sum(1, keepdim=True, dtype=torch.float64)
    lse = top.double() + total.log()
    return keep, label, e, total, (z_label - lse)[:, 0], lse[:, 0]


def _plain_gradient(s, keep, label, e, total, at_label, everywhere):
    """scale * (at_label * onehot + everywhere * softmax), 0 in the rows that are not kept."""
    zero = torch.zeros_like(total)
    d = e.mul_((torch.where(keep[:, None], everywhere[:, None], zero) / total).float() * s["scale"])
    d.scatter_add_(1, label, (torch.where(keep[:, None], at_label[:, None], zero) * s["scale"]).float())
    return d.to(s["logits"].dtype)


def _plain_logits(s):
    kind = s["case"]["kind"]
    keep, label, e, total, logp, lse = _plain_rows(s)
    zero = torch.zeros_like(logp)
    if kind == "logp_bwd":
        a, b = s["dlogp"].double(), s["dlse"].double()
        return {"dlogits": _plain_gradient(s, keep, label, e, total, a, b - a)}
    out = {"logp": torch.where(keep, logp, zero).float()}
    if kind == "logp_fwd":
        return {**out, "lse": torch.where(keep, lse, zero).float()}
    c = s["reduce"] * (1.0 if s["weight"] is None else s["weight"].double())
    if kind == "token_loss":
        z_term = torch.where(keep, c * s["z_coef"] * lse * lse, zero)
        loss = torch.where(keep, -c * logp, zero) + z_term
        out["lse"] = torch.where(keep, lse, zero).float()
        out["stats"] = torch.stack([loss.sum(), z_term.sum()]).float()
        g = c + zero
        out["dlogits"] = _plain_gradient(s, keep, label, e, total, -g, g + 2 * s["z_coef"] * lse * c)
        return out
    a = s["advantage"].double()
    ratio = torch.ones_like(logp) if s["old"] is None else (logp - s["old"].double()).exp()
    low, high = 1.0 - s["low"], 1.0 + s["high"]
    clipped = torch.where(a > 0, ratio > high, (ratio < low) & (a < 0))
    loss = -torch.minimum(ratio * a, ratio.clamp(low, high) * a)
    g = torch.where(clipped, zero, -a * ratio)
    kl = zero
    if s["ref"] is not None:
        q = s["ref"].double() - logp
        kl = q.exp() - q - 1.0
        loss = loss + s["kl"] * kl
        g = g + s["kl"] * (1.0 - q.exp())
    out["stats"] = torch.stack([torch.where(keep, c * x, zero).sum() for x in (loss, kl, clipped.double())]).float()
    out["dlogits"] = _plain_gradient(s, keep, label, e, total, c * g, -c * g)
    return out


def _plain_preference(s):
    offsets = s["offsets"].long()
    lengths = offsets[1:] - offsets[:-1]
    pairs = len(lengths) // 2
    diff = s["logp"].double() - (0.0 if s["ref"] is None else s["ref"].double())
    run_sum = torch.cat([diff.new_zeros(1), diff.cumsum(0)])
    sums = (run_sum[offsets[1:]] - run_sum[offsets[:-1]]).view(pairs, 2)
    z = s["beta"] * (sums[:, 0] - sums[:, 1])
    # log(1 + exp(-z)) without overflow
    soft = torch.log1p(torch.exp(-z.abs()))
    loss = (1.0 - s["smoothing"]) * (soft + (-z).clamp_min(0)) + s["smoothing"] * (soft + z.clamp_min(0))
    sigma = 1.0 / (1.0 + torch.exp(-z))
    g = (-(1.0 - s["smoothing"]) * (1.0 - sigma) + s["smoothing"] * sigma) * s["beta"] / pairs
    dlogp = torch.repeat_interleave(torch.stack([g, -g], 1).reshape(-1), lengths, output_size=len(diff))
    return {"stats": torch.stack([loss.mean(), (z > 0).double().mean(), z.mean()]).float(), "margin": z.float(), "dlogp": dlogp.float()}


_WORD = 0xFFFFFFFF


def _mix(x):
    """32 bits mixed, in 64-bit integers."""
    x = ((x ^ (x >> 16)) * 0x6A09E667) & _WORD
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & _WORD
    return x ^ (x >> 16)


def _plain_values(code, scale, mantissa):
    """What codes of magnitudes with 4 exponent bits stand for."""
    e, f = (code >> mantissa).int(), (code & (2 ** mantissa - 1)).float()
    return torch.where(e > 0, (f + 2 ** mantissa) * torch.exp2((e - 1).float()), f) * scale


def _plain_codes(x, mantissa, top, draw_bits):
    """Rounded up with the probability of the distance to the lower code, by 16 random bits."""
    scale = x.amax(1, keepdim=True) / top
    y = x / torch.where(scale > 0, scale, 1.0)
    shift = 23 - mantissa
    high = ((y.view(torch.int32) + (draw_bits << (shift - 16)).int()) >> shift) - ((126 + mantissa) << mantissa)
    low = torch.floor(y + draw_bits.float() / 65536.0).int()
    return torch.where(y >= 2 ** mantissa, high, low).clamp_max_(2 ** (mantissa + 4) - 1), scale


def _plain_update(s):
    case = s["case"]
    total = len(s["m"])
    shift = 1 if case["odd"] else 0
    p, g = (s[k][shift:shift + total].view(-1, BLOCK) for k in ("p", "g"))
    factor = 1.0 if s["norm"] is None else (s["max_norm"] / s["norm"].double()).clamp_max(1.0).float()
    g = g.float() * factor
    if case["bits"] == 8:
        code_m, code_v = s["m"].view(-1, BLOCK), s["v"].view(-1, BLOCK)
        m = _plain_values(code_m & 127, s["m_scale"][:, None], 3)
        m = torch.where(code_m > 127, -m, m)
        v = _plain_values(code_v, s["v_scale"][:, None], 4)
    else:
        m, v = s["m"].view(-1, BLOCK), s["v"].view(-1, BLOCK)
    s["step"] += 1
    t = s["step"].double()
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * g * g
    rate = (RATE / (1.0 - BETA1 ** t)).float()
    root = (1.0 / (1.0 - BETA2 ** t)).sqrt().float()
    new = p.float() * (1.0 - RATE * s["decay"]).float()[:, None] - rate * (m / (v.sqrt() * root + EPS))
    p.copy_(new)
    if s["copy"] is not None:
        s["copy"][shift:shift + total].view(-1, BLOCK).copy_(new)
    out = {"p": s["p"], "step": s["step"]}
    if s["copy"] is not None:
        out["copy"] = s["copy"]
    if case["bits"] == 32:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
        return {**out, "m": s["m"], "v": s["v"]}
    key = _mix(_mix(_mix(s["step"] & _WORD) + s["number"] & _WORD))
    index = (torch.arange(len(m), device="cuda") - s["first"])[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    bits = _mix(index + key[:, None] & _WORD)
    code, scale = _plain_codes(m.abs(), 3, 245760.0, bits & 0xFFFF)
    s["m"].copy_((code | (m < 0).int() << 7).view(-1))
    s["m_scale"].copy_(scale[:, 0])
    out["m"] = torch.where(m < 0, -_plain_values(code, scale, 3), _plain_values(code, scale, 3)).to(torch.bfloat16).view(-1)
    code, scale = _plain_codes(v, 4, 507904.0, bits >> 16)
    code = torch.maximum(code, (v > 0).int())
    s["v"].copy_(code.view(-1))
    s["v_scale"].copy_(scale[:, 0])
    out["v"] = _plain_values(code, scale, 4).to(torch.bfloat16).view(-1)
    return out


def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    if kind == "preference":
        return _plain_preference(s)
    return _plain_update(s) if kind == "adamw" else _plain_logits(s)


# ---- what a call cannot do without -------------------------------------------------


def work(case):
    """Inputs read once, outputs written once."""
    kind = case["kind"]
    if kind == "preference":
        n = case["pairs"] * (2 * case["length"] + 1)
        return {"bytes": n * (12 if case["ref"] else 8) + case["pairs"] * (20 if case["offsets"] == "i64" else 12), "flops": 3 * n}
    if kind == "adamw":
        n = sum(k for k, _ in _lengths(case))
        per = (4 if case["params"] == "bf16" else 8) + (2 if case["params"] == "f32+copy" else 0) + (2 if case["grads"] == "bf16" else 4)
        # states read and written; in 8 bits with their scales, and read out as bf16 values
        per += 16 if case["bits"] == 32 else 2 * (2 + 8 / BLOCK) + 2 * 2
        return {"bytes": per * n, "flops": (16 if case["bits"] == 32 else 60) * n}
    t, v = case["tokens"], case["vocab"]
    size = 4 if case["dtype"] == "f32" else 2
    kept = t * (1 - case["padding"]) * (0.84 if case.get("weights") else 1.0)      # tokens whose logits count
    bytes_ = kept * v * size + t * (4 if case["ids"] == "i32" else 8)
    if kind != "logp_fwd":
        bytes_ += t * v * size
    rows = {"logp_fwd": 8, "logp_bwd": 12, "token_loss": 8 + (4 if case.get("weights") else 0),
            "policy": 12 + (4 if case.get("old") else 0) + (4 if case.get("kl") else 0)}[kind]
    return {"bytes": bytes_ + rows * t, "flops": (4 if kind == "logp_fwd" else 7) * kept * v}


# ---- 64 bits ------------------------------------------------------------------------


def _exact_logits(case, seed):
    i = _logit_inputs(case, seed)
    kind, v, scale = case["kind"], case["vocab"], case["scale"]
    ids = i["ids"].long()
    on = ids >= 0
    w = torch.ones(len(ids), dtype=torch.float64, device="cuda")
    if i.get("weight") is not None:
        w = i["weight"].double()
        on = on & (w > 0)
    w = w * i["reduce"] * on
    row = {k: i[k].double() for k in ("dlogp", "dlse", "advantage", "old", "ref") if i.get(k) is not None}
    logp, lse = torch.zeros_like(w), torch.zeros_like(w)
    grad = None if kind == "logp_fwd" else torch.empty((len(ids), v), dtype=torch.float64, device="cuda")
    terms = torch.zeros((len(ids), 3), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 28) // v)
    for a in range(0, len(ids), step):
        part = slice(a, a + step)
        z = torch.log_softmax(i["logits"][part].double() * scale, 1)
        live = on[part]
        at = torch.where(live, ids[part], 0)[:, None]
        lp = z.gather(1, at)[:, 0]
        first = i["logits"][part].double().gather(1, at)[:, 0] * scale
        ls = first - lp
        logp[part], lse[part] = torch.where(live, lp, 0.0), torch.where(live, ls, 0.0)
        if grad is None:
            continue
        c = w[part]
        if kind == "logp_bwd":
            one, all_ = row["dlogp"][part] * live, (row["dlse"] - row["dlogp"])[part] * live
        elif kind == "token_loss":
            terms[part, 1] = c * i["z_coef"] * ls ** 2
            terms[part, 0] = terms[part, 1] - c * lp
            one, all_ = -c, c * (1.0 + 2.0 * i["z_coef"] * ls)
        else:
            adv = row["advantage"][part]
            r = torch.exp(lp - row["old"][part]) if "old" in row else torch.ones_like(lp)
            inside = torch.where(adv >= 0, r <= 1.0 + i["high"], r >= 1.0 - i["low"])
            bounded = torch.where(adv >= 0, r.clamp_max(1.0 + i["high"]), r.clamp_min(1.0 - i["low"]))
            one = -adv * r * inside
            terms[part, 0], terms[part, 2] = -adv * bounded * c, c * ~inside
            if "ref" in row:
                x = row["ref"][part] - lp
                terms[part, 1] = c * (torch.expm1(x) - x)
                terms[part, 0] += i["kl"] * terms[part, 1]
                one = one - i["kl"] * torch.expm1(x)
            one = one * c
            all_ = -one
        g = z.exp_().mul_((all_ * scale)[:, None])
        g.scatter_add_(1, at, (one * scale)[:, None])
        grad[part] = torch.where(live[:, None], g, 0.0)
    out = {} if kind == "logp_bwd" else {"logp": logp}
    if kind in ("logp_fwd", "token_loss"):
        out["lse"] = lse
    if grad is not None:
        out["dlogits"] = grad
    if kind == "token_loss":
        out["stats"] = terms[:, :2].sum(0)
    elif kind == "policy":
        out["stats"] = terms.sum(0)
    return out


def _exact_preference(case, seed):
    i = _pair_inputs(case, seed)
    of = i["offsets"].cpu().tolist()
    x = i["logp"].double() - (i["ref"].double() if i["ref"] is not None else 0.0)
    sums = torch.stack([p.sum() for p in x.cpu().split([b - a for a, b in zip(of, of[1:])])]).view(-1, 2)
    z = i["beta"] * (sums[:, 0] - sums[:, 1])
    q = i["smoothing"]
    loss = -(1 - q) * torch.nn.functional.logsigmoid(z) - q * torch.nn.functional.logsigmoid(-z)
    dz = (q - torch.sigmoid(-z)) * i["beta"] / len(z)
    dlogp = torch.cat([d.expand(n) for d, n in zip(torch.stack([dz, -dz], 1).reshape(-1), [b - a for a, b in zip(of, of[1:])])])
    return {"stats": torch.stack([loss.mean(), (z > 0).double().mean(), z.mean()]), "margin": z, "dlogp": dlogp}


def _exact_bits(x):
    """The same mixing in wrapping 32-bit integers."""
    def down(y, k):
        return (y >> k) & ((1 << (32 - k)) - 1)

    x = (x ^ down(x, 16)) * 0x6A09E667
    x = (x ^ down(x, 15)) * (0xBB67AE85 - (1 << 32))
    return x ^ down(x, 16)


def _exact_states(x, mantissa, top, u):
    """What the states hold after their rounding: y in units of its binade's step, with ``u`` added, cut off."""
    scale = x.amax(1, keepdim=True) / top
    y = torch.where(scale > 0, x / scale, 0.0)
    unit = torch.ldexp(torch.ones_like(y), (torch.frexp(y)[1] - 1 - mantissa).clamp_min(0))
    return torch.floor(y / unit + u).mul_(unit).clamp_max_(top), scale


def _exact_update(case, seed):
    i = _update_inputs(case, seed)
    total = len(i["m"])
    shift = 1 if case["odd"] else 0
    number, decay, first = _tensor_of_block(case)
    p, g = (i[k][shift:shift + total].view(-1, BLOCK).double() for k in ("p", "g"))
    if case["clip"]:
        g *= min(1.0, i["max_norm"] / float(i["norm"]))
    if case["bits"] == 8:
        def read(code, mantissa, scale):
            table = [k if k < 2 ** mantissa else (k % 2 ** mantissa + 2 ** mantissa) << (k >> mantissa) - 1 for k in range(2 ** (mantissa + 4))]
            return torch.tensor(table, dtype=torch.float64, device="cuda")[code.long()].view(-1, BLOCK) * scale.double()[:, None]

        m, v = read(i["m"] % 128, 3, i["m_scale"]), read(i["v"], 4, i["v_scale"])
        m *= 1.0 - 2.0 * (i["m"].view(-1, BLOCK) // 128)
    else:
        m, v = (i[k].view(-1, BLOCK).double() for k in ("m", "v"))
    t = int(i["step"]) + 1
    m, v = m + (1 - BETA1) * (g - m), v + (1 - BETA2) * (g * g - v)
    p = p - RATE * (decay[:, None] * p + (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)) ** 0.5 + EPS))
    if case["bits"] == 8:
        word = torch.tensor([t], dtype=torch.int32, device="cuda")
        key = _exact_bits(_exact_bits(_exact_bits(word) + number.int()))
        place = (torch.arange(len(m), device="cuda") - first)[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
        bits = _exact_bits(place.int() + key[:, None])
        held, scale = _exact_states(m.abs(), 3, 245760.0, (bits & 0xFFFF).double() / 65536)
        m = torch.sign(m) * held * scale
        held, scale = _exact_states(v, 4, 507904.0, (bits >> 16 & 0xFFFF).double() / 65536)
        v = torch.where(v > 0, held.clamp_min(1.0), 0.0) * scale

    def whole(x):
        flat = torch.zeros(total + 8, dtype=torch.float64, device="cuda")
        flat[shift:shift + total] = x.reshape(-1)
        return flat

    out = {"p": whole(p), "step": i["step"] + 1, "m": m.reshape(-1), "v": v.reshape(-1)}
    if i["copy"] is not None:
        out["copy"] = whole(p)
    return out


def exact(case, seed):
    if case["kind"] == "preference":
        return _exact_preference(case, seed)
    return _exact_update(case, seed) if case["kind"] == "adamw" else _exact_logits(case, seed)
