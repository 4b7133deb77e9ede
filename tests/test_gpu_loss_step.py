"""The loss and the update as a training step uses them together: logits to losses, their
gradient to the weights' and to AdamW with the gradients' norm, against the same steps in
64-bit torch; the calls captured in a graph, and made on another stream."""
import numpy as np
import pytest
import torch

import paper_2605_03667_amd as elas
from examples.train_stack import Stack

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


class _Head:
    """Logits of a linear layer over fixed features, trained by every loss in turn: tokens, then a policy on
    sampled ones, then pairs of answers."""

    def __init__(self, bits, T=600, V=1111, d=64, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
        self.w, self.b = rand(V, d) * 0.1, rand(V) * 0.1
        self.copies = [torch.empty_like(t, dtype=BF) for t in (self.w, self.b)]
        self.grads = [torch.zeros_like(t) for t in (self.w, self.b)]
        self.opt = elas.ElasAdamW([self.w, self.b], copies=self.copies, decay=[0.1, 0.0], bits=bits)
        self.list = elas.ElasTensors(self.grads)
        self.x = rand(T, d)
        self.ids = torch.randint(-1, V, (T,), generator=g, device=DEV)
        self.weight, self.advantage = rand(T).abs(), rand(T)
        self.offsets = torch.tensor([0, 100, 200, 333, 334, 600, 600], device=DEV)
        self.logits = torch.empty((T, V), device=DEV)
        self.old, self.ref = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        self.out = {"token": {"stats": torch.empty(2, device=DEV), "logp": torch.empty(T, device=DEV), "lse": torch.empty(T, device=DEV)},
                    "policy": {"stats": torch.empty(3, device=DEV), "logp": torch.empty(T, device=DEV)},
                    "logp": {"logp": torch.empty(T, device=DEV), "lse": torch.empty(T, device=DEV)},
                    "pairs": {"stats": torch.empty(3, device=DEV), "margin": torch.empty(3, device=DEV), "dlogp": torch.empty(T, device=DEV)}}
        self.norm = torch.empty(1, device=DEV)
        self.ws = {"loss": torch.empty(elas.elas_token_loss_workspace_bytes(T, V, elas.ELAS_LOGITS_F32), dtype=torch.uint8, device=DEV),
                   "pairs": torch.empty(elas.elas_preference_loss_workspace_bytes(T, 3), dtype=torch.uint8, device=DEV),
                   "grad": torch.empty(elas.elas_grad_workspace_bytes(2), dtype=torch.uint8, device=DEV)}

    def forward(self):
        torch.addmm(self.b, self.x, self.w.t(), out=self.logits)

    def update(self):
        """From the logits' gradient, which lies over them."""
        torch.mm(self.logits.t(), self.x, out=self.grads[0])
        torch.sum(self.logits, 0, out=self.grads[1])
        elas.elas_grad_norm(self.list, norm=self.norm, workspace=self.ws["grad"])
        elas.elas_adamw_step(self.opt, self.list, 1e-2, norm=self.norm, max_norm=0.5, beta2=0.95)

    def token(self):
        elas.elas_token_loss(self.logits, self.ids, weight=self.weight, reduce=1 / 600, z_coef=1e-3, out={**self.out["token"], "dlogits": self.logits},
                             workspace=self.ws["loss"])
        self.old.copy_(self.out["token"]["logp"])
        self.ref.copy_(self.out["token"]["logp"])

    def policy(self):
        elas.elas_policy_loss(self.logits, self.ids, self.advantage, old_logp=self.old, ref_logp=self.ref, reduce=1 / 600, kl_coef=0.1,
                              out={**self.out["policy"], "dlogits": self.logits}, workspace=self.ws["loss"])

    def pairs(self):
        elas.elas_token_logp_fwd(self.logits, self.ids, out=self.out["logp"])
        elas.elas_preference_loss(self.out["logp"]["logp"], self.offsets, ref_logp=self.ref, beta=0.3, smoothing=0.1, out=self.out["pairs"],
                                  workspace=self.ws["pairs"])
        elas.elas_token_logp_bwd(self.out["pairs"]["dlogp"], self.logits, self.ids, self.out["logp"]["lse"], dlogits=self.logits)

    def run(self):
        for loss in (self.token, self.policy, self.pairs):
            self.forward()
            loss()
            self.update()

    def state(self):
        return [self.w, self.b, *self.copies, *self.grads, self.opt.m, self.opt.v, self.opt.step, self.norm, self.old,
                *(t for o in self.out.values() for t in o.values())]


def _reference(h):
    """The same three steps by 64-bit autograd, with the library's update formula: weights and statistics."""
    w, b = (t.double().clone().requires_grad_() for t in (h.w, h.b))
    m, v = [torch.zeros_like(t) for t in (w, b)], [torch.zeros_like(t) for t in (w, b)]
    on = h.ids >= 0
    at = h.ids.clamp_min(0)[:, None]
    stats, kept = [], []

    def logp():
        z = h.x.double() @ w.t() + b
        lse = torch.logsumexp(z, 1)
        return torch.where(on, z.gather(1, at)[:, 0] - lse, 0.0), torch.where(on, lse, 0.0)

    def step(loss, t):
        for p in (w, b):
            p.grad = None
        loss.backward()
        norm = torch.sqrt(sum((p.grad ** 2).sum() for p in (w, b)))
        f = min(1.0, 0.5 / float(norm))
        with torch.no_grad():
            for k, (p, decay) in enumerate(((w, 0.1), (b, 0.0))):
                g = p.grad * f
                m[k] = 0.9 * m[k] + 0.1 * g
                v[k] = 0.95 * v[k] + 0.05 * g * g
                p -= 1e-2 * (decay * p + m[k] / (1 - 0.9 ** t) / (torch.sqrt(v[k] / (1 - 0.95 ** t)) + 1e-8))

    lp, lse = logp()
    loss = (h.weight.double() * on * (1e-3 * lse ** 2 - lp)).sum() / 600
    stats.append(loss.item())
    kept = lp.detach()
    step(loss, 1)
    lp, _ = logp()
    r, q, a = torch.exp(lp - kept), kept - lp, h.advantage.double()
    loss = (on * (-torch.minimum(r * a, r.clamp(0.8, 1.2) * a) + 0.1 * (torch.exp(q) - q - 1))).sum() / 600
    stats.append(loss.item())
    step(loss, 2)
    lp, _ = logp()
    o = h.offsets.tolist()
    sums = torch.stack([(lp - kept)[i:j].sum() for i, j in zip(o, o[1:])]).view(-1, 2)
    z = 0.3 * (sums[:, 0] - sums[:, 1])
    loss = (-0.9 * torch.nn.functional.logsigmoid(z) - 0.1 * torch.nn.functional.logsigmoid(-z)).mean()
    stats.append(loss.item())
    step(loss, 3)
    return w.detach(), b.detach(), stats


def test_three_steps_against_autograd():
    """The weights move by about the rate a step whatever the gradient's size, and where a gradient is
    near 0 against its rounding (2^-24 of terms 10^3 times its size at most) the direction is uncertain: 1e-3 of the
    distance moved is allowed over all, and 2e-5 of a loss (float32 logits of 2^-24 sqrt(64) relative error)."""
    h = _Head(32)
    start = h.w.clone()
    w, b, stats = _reference(h)
    h.run()
    assert torch.linalg.norm(h.w - w) <= 1e-3 * torch.linalg.norm(start - w)
    got = [float(h.out[k]["stats"][0]) for k in ("token", "policy", "pairs")]
    for g, s in zip(got, stats):
        assert abs(g - s) <= 2e-5 * max(1.0, abs(s)), (got, stats)
    assert torch.equal(h.copies[0], h.w.to(BF)) and torch.equal(h.copies[1], h.b.to(BF))


@pytest.mark.parametrize("bits", [32, 8])
def test_graph_replays_match_eager(bits):
    """Library products and sums in the graph are torch's; the sum over rows is done by a product here, since
    torch's own may record a memory clear."""
    def make():
        h = _Head(bits, seed=3)
        ones = torch.ones((1, 600), device=DEV)

        def update():
            torch.mm(h.logits.t(), h.x, out=h.grads[0])
            torch.mm(ones, h.logits, out=h.grads[1].view(1, -1))
            elas.elas_grad_norm(h.list, norm=h.norm, workspace=h.ws["grad"])
            elas.elas_adamw_step(h.opt, h.list, 1e-2, norm=h.norm, max_norm=0.5, beta2=0.95)

        h.update = update
        return h

    eager, captured = make(), make()
    begin = [t.clone() for t in captured.state()]
    scales = [captured.opt.m_scale, captured.opt.v_scale] if bits == 8 else []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        captured.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for t, b in zip(captured.state(), begin):
        t.copy_(b)
    for t in scales:
        t.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    for rep in range(4):
        eager.run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, (a, b) in enumerate(zip(eager.state(), captured.state())):
            assert torch.equal(a, b), (rep, k)
    assert int(captured.opt.step) == 12


def test_other_stream():
    """The calls go to torch's current stream: work queued there before them is seen."""
    a, b = _Head(8, seed=1), _Head(8, seed=1)
    a.run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for t in (b.logits, b.old, *b.grads):
            t.fill_(3.0)
        b.run()
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.state(), b.state()))


def test_two_streams_at_once():
    """Calls in flight together, each with its own workspace (allocated for its stream)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = torch.randn((4000, 5000), generator=g, device=DEV).to(BF)
    ids = torch.randint(0, 5000, (4000,), generator=g, device=DEV)
    want = [elas.elas_token_loss(x, ids), elas.elas_token_loss(x, ids.flip(0))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(3):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(elas.elas_token_loss(x, ids if k == 0 else ids.flip(0)))
    torch.cuda.synchronize()
    for k in range(2):
        for r in got[k]:
            assert all(torch.equal(r[n], want[k][n]) for n in r)


@pytest.mark.parametrize("T", [12, 700])
def test_two_graphs_with_one_workspace(T):
    """Replayed in turn, with other calls on the same workspace between (12 rows are split over workgroups)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    V = 20000
    x = torch.randn((T, V), generator=g, device=DEV).to(BF)
    ids = torch.randint(-1, V, (T,), generator=g, device=DEV)
    adv = torch.randn(T, generator=g, device=DEV)
    ws = torch.empty(elas.elas_token_loss_workspace_bytes(T, V), dtype=torch.uint8, device=DEV)
    outs = [{"stats": torch.empty(k, device=DEV), "logp": torch.empty(T, device=DEV), "dlogits": torch.empty_like(x)} for k in (2, 3)]
    calls = [lambda: elas.elas_token_loss(x, ids, z_coef=0.1, out=outs[0], workspace=ws), lambda: elas.elas_policy_loss(x, ids, adv, out=outs[1], workspace=ws)]
    want, graphs = [], []
    for call, out in zip(calls, outs):
        call()
        want.append({k: t.clone() for k, t in out.items()})
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
    for rep in range(3):
        for out in outs:
            for t in out.values():
                t.fill_(9.0)
        for graph in graphs:
            graph.replay()
        elas.elas_token_loss(x, ids, out={"stats": torch.empty(2, device=DEV)}, workspace=ws)
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            assert all(torch.equal(out[k], w[k]) for k in w), rep


def test_timing_tags():
    h = _Head(8)
    try:
        elas.elas_timing_enable(True)
        h.run()
        elas.elas_adam8_values(h.opt.m, h.opt.m_scale)
        elas.elas_preference_loss(h.old, torch.arange(201, device=DEV))       # (few pairs take one launch)
        torch.cuda.synchronize()
        elas.elas_timing_enable(False)
        tags = elas.elas_timing_collect()
    finally:
        elas.elas_timing_enable(False)
    assert {"token_logp", "token_logp_bwd", "token_loss", "policy_loss", "loss_sum", "preference", "preference_sum", "adamw_factors", "adamw8",
            "adam8_values", "grad_square", "grad_norm"} == set(tags)
    assert tags["adamw8"][0] == 3 and all(ms > 0 for _, ms in tags.values())


def test_debug_sync_same_results():
    a, b = _Head(8, seed=2), _Head(8, seed=2)
    a.run()
    prev = elas.elas_debug_sync(True)
    try:
        b.run()
    finally:
        elas.elas_debug_sync(prev)
    assert all(torch.equal(x, y) for x, y in zip(a.state(), b.state()))


def test_example_gradients():
    """The example's gradients of its loss, against float32 autograd of the same stack at its bf16 weights (dense
    activations).  Between the two lie the bf16 roundings of the block's intermediate values, of the logits and of their
    gradient, about a dozen a block of relative size 2^-9 each: a percent; 3 % is allowed."""
    model = Stack(300, 256, 344, 64, 2, seed=3, mode=elas.ELAS_MODE_DENSE)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    ids, targets = (torch.randint(0, 300, (777,), generator=g, device=DEV) for _ in range(2))
    n, saved = model.forward(ids)
    stats, dn = model.loss(n, targets)
    model.backward(dn, saved)

    w = {k: v.float().requires_grad_() for k, v in [*model.w.items(), ("head", model.head)]}

    def norm(v, gain):
        return v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6) * gain

    h = w["table"][ids] * model.d ** 0.5
    for k in range(model.layers):
        s = torch.relu(norm(h, w[f"{k}.w_pre"]) @ w[f"{k}.U_up"] @ w[f"{k}.V_up"]).square()
        h = h + model.block_scale * w[f"{k}.gate"] * norm(s @ w[f"{k}.U_down"] @ w[f"{k}.V_down"], w[f"{k}.w_post"])
    z = norm(h, w[f"{model.layers}.w_pre"]) @ w["head"].t()
    lse = torch.logsumexp(z, 1)
    loss = (lse - z[torch.arange(777), targets] + 1e-4 * lse ** 2).mean()
    loss.backward()
    assert abs(float(stats[0]) - loss.item()) < 0.01 * loss.item()
    for k, grad in [*model.grad.items(), ("head", model.head_grad)]:
        assert torch.linalg.norm(grad - w[k].grad) < 0.03 * torch.linalg.norm(w[k].grad), k


@pytest.mark.parametrize("bits", [32, 8])
def test_example_step(bits):
    """A step of the example changes every weight by at most about the rate (AdamW's first step moves a value by
    the rate where its gradient is above eps, and by the decay), and writes the copies of the new weights."""
    model = Stack(200, 128, 344, 64, 2, seed=1, bits=bits)
    before = {k: v.clone() for k, v in model.master.items()}
    ids = torch.randint(0, 200, (512,), device=DEV)
    n, saved = model.forward(ids)
    _, dn = model.loss(n, ids.flip(0))
    model.backward(dn, saved)
    norm = model.update(1e-2, 1.0)
    assert torch.isfinite(norm).all() and int(model.opt.step) == 1
    for k, v in model.master.items():
        moved = (v - before[k]).abs()
        assert moved.max() > 0 and (moved <= 1e-2 * (1.001 + 0.1 * before[k].abs()) + 2.0 ** -23 * before[k].abs()).all(), k
        assert torch.equal(model.w[k], v.to(BF)), k


@pytest.mark.parametrize("change, match", [(lambda t: t.t(), "contiguous"), (lambda t: t.view(torch.int32), "float32 or torch.bfloat16"),
                                           (lambda t: t.to(BF), None), (lambda t: t[:2], None), (lambda t: t.reshape(4, 8), None)])
def test_a_handle_in_use_sees_what_its_tensors_became(change, match):
    """After several steps with the same tensors, one is given another type, length or order, in the same memory or not."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    ts = [torch.randn((8, 4), generator=gen, device=DEV) for _ in range(3)]
    h = elas.ElasTensors(ts)
    want = elas.elas_grad_norm(h).clone()
    for mode in (torch.enable_grad, torch.no_grad, torch.inference_mode, torch.enable_grad):
        with mode():
            assert torch.equal(elas.elas_grad_norm(h), want)
    before = ts[1].data
    ts[1].data = change(before)
    if match:
        for _ in range(2):
            with pytest.raises(ValueError, match=match):
                elas.elas_grad_norm(h)
    else:
        for _ in range(3):
            assert torch.equal(elas.elas_grad_norm(h), elas.elas_grad_norm([t.clone() for t in ts]))
    ts[1].data = before
    for _ in range(3):
        assert torch.equal(elas.elas_grad_norm(h), want)


def test_a_handle_may_hold_a_tensor_twice():
    g = torch.full((100,), 2.0, device=DEV)
    h = elas.ElasTensors([g, g])
    for _ in range(4):
        assert float(elas.elas_grad_norm(h)) == np.float32(800.0 ** 0.5)
