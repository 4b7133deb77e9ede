"""The operators around the FFN as a training step uses them together: the
example's gradients against float32 autograd of the same stack, its loss, and
the calls captured in a graph and made on another stream."""
import pytest
import torch

import paper_2605_03667_amd as elas
from examples.train_stack import Stack, train

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _autograd(model, ids, dn):
    """Gradients of sum(n dn) by torch, in float32, at the model's bf16 weights."""
    w = {k: v.float().requires_grad_() for k, v in model.w.items()}

    def norm(v, gain):
        return v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6) * gain

    h = w["table"][ids] * model.d ** 0.5
    for k in range(model.layers):
        x = norm(h, w[f"{k}.w_pre"])
        s = torch.relu(x @ w[f"{k}.U_up"] @ w[f"{k}.V_up"]).square()
        y = s @ w[f"{k}.U_down"] @ w[f"{k}.V_down"]
        h = h + model.block_scale * w[f"{k}.gate"] * norm(y, w[f"{k}.w_post"])
    n = norm(h, w[f"{model.layers}.w_pre"])
    (n * dn.float()).sum().backward()
    return n.detach(), {k: v.grad for k, v in w.items()}


def test_gradients_of_the_stack():
    """Dense activations, so that autograd computes the same function.  Between two
    float32 chains lie the bf16 roundings of P, H, S, Z, y and n and of their
    gradients, about ten a block of relative size 2^-9 each: relative errors of a
    few 2^-9 sqrt(10 L) = 1 %; 3 % is allowed."""
    model = Stack(300, 256, 344, 64, 2, seed=3, mode=elas.ELAS_MODE_DENSE)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(5)
    ids = torch.randint(0, 300, (777,), generator=gen, device=DEV)
    dn = torch.randn((777, 256), generator=gen, device=DEV).to(BF)
    n, saved = model.forward(ids)
    model.backward(dn, saved)
    n_ref, ref = _autograd(model, ids, dn)
    assert torch.linalg.norm(n.float() - n_ref) < 0.03 * torch.linalg.norm(n_ref)
    for k, g in model.grad.items():
        assert torch.linalg.norm(g - ref[k]) < 0.03 * torch.linalg.norm(ref[k]), k


def test_example_learns():
    losses = train(steps=60, tokens=2048, layers=2, vocab=200, d=128, d_ff=344, r=64)
    assert all(v == v for v in losses)
    assert losses[-1] < 0.7 * losses[0], (losses[0], losses[-1])


def _step_calls():
    """A closure over fixed tensors that makes every call once, and its outputs."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    T, d, V = 4500, 768, 5000

    def rand(*shape, dtype=BF):
        return torch.randn(shape, generator=g, device=DEV).to(dtype)

    ids = torch.randint(-1, V, (T,), generator=g, device=DEV)
    table, b, gate, w1, w2, dn = rand(V, d), rand(T, d), rand(d), rand(d), rand(d), rand(T, d)
    out = {"x": torch.empty((T, d), dtype=BF, device=DEV), "h": torch.empty((T, d), dtype=BF, device=DEV),
           "n": torch.empty((T, d), dtype=BF, device=DEV), "dh": torch.empty((T, d), dtype=BF, device=DEV),
           "db": torch.empty((T, d), dtype=BF, device=DEV), "table": torch.empty((V, d), device=DEV),
           "stats": torch.empty(2, device=DEV), "norm": torch.empty(1, device=DEV)}
    for k in ("dgate", "dw_post", "dw_pre"):
        out[k] = torch.empty(d, device=DEV)
    sums = [out[k] for k in ("table", "dgate", "dw_post", "dw_pre")]
    clipped = [torch.empty_like(t) for t in sums]
    grads, to = elas.ElasTensors(sums), elas.ElasTensors(clipped)
    ws = {"join": elas.elas_norm_join_bwd_workspace_bytes(T, d), "embed": elas.elas_embed_bwd_workspace_bytes(T, V, d, elas.ELAS_IDS_I64),
          "grad": elas.elas_grad_workspace_bytes(4)}
    ws = {k: torch.empty(v, dtype=torch.uint8, device=DEV) for k, v in ws.items()}

    def step():
        elas.elas_embed_fwd(ids, table, 2.0, out=out["x"])
        elas.elas_norm_join_fwd(out["x"], b, gate, w1, w2, out=out)
        elas.elas_norm_join_bwd(None, dn, out["h"], b, gate, w1, w2, grads=out, workspace=ws["join"])
        elas.elas_embed_bwd(ids, out["dh"], V, 2.0, dtable=out["table"], workspace=ws["embed"])
        elas.elas_grad_norm(grads, norm=out["norm"], workspace=ws["grad"])
        elas.elas_grad_clip(grads, 1.0, out=to, stats=out["stats"], workspace=ws["grad"])

    return step, [*out.values(), *clipped]


def test_graph_replays_match_eager():
    step, outs = _step_calls()
    step()
    torch.cuda.synchronize()
    ref = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(3):
        for t in outs:
            t.zero_()                     # eager work between the replays
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, r) for t, r in zip(outs, ref)), rep


def test_other_stream():
    """The calls go to torch's current stream: work queued there before them is seen."""
    step, outs = _step_calls()
    step()
    torch.cuda.synchronize()
    ref = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for t in outs:
            t.fill_(3.0)
        step()
    side.synchronize()
    assert all(torch.equal(t, r) for t, r in zip(outs, ref))


def test_timing_tags():
    step, _ = _step_calls()
    try:
        elas.elas_timing_enable(True)
        step()
        torch.cuda.synchronize()
        elas.elas_timing_enable(False)
        tags = elas.elas_timing_collect()
    finally:
        elas.elas_timing_enable(False)
    assert set(tags) == {"embed_fwd", "norm_join_fwd", "norm_join_bwd", "norm_join_bwd_sums", "embed_bwd_sort", "embed_bwd_sum", "embed_bwd_join",
                         "grad_square", "grad_norm", "grad_scale"}
    assert tags["grad_square"][0] == 2 and all(ms > 0 for _, ms in tags.values())


def test_debug_sync_same_results():
    step, outs = _step_calls()
    step()
    torch.cuda.synchronize()
    ref = [t.clone() for t in outs]
    prev = elas.elas_debug_sync(True)
    try:
        step()
    finally:
        elas.elas_debug_sync(prev)
    assert all(torch.equal(t, r) for t, r in zip(outs, ref))
