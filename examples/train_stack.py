"""Trains a small stack of ELAS blocks with the operators around them, as a
training step uses them together:

    ids -> embedding -> [norm -> low-rank 2:4 FFN -> norm, gate, residual sum] x L
        -> norm -> loss -> the same backward -> clipping -> update

    python examples/train_stack.py [--steps N] [--tokens T] [--layers L]

Each token learns to predict a fixed vector of the token that follows it (a
permutation of the vocabulary), so no sequence mixing is needed.  torch provides
the memory, the squared-error loss and the update of the float32 master weights;
everything between is libelas.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_03667_amd as elas  # noqa: E402

BF = torch.bfloat16


class Stack:
    """Weights of the stack: float32 masters, their bf16 copies and gradients."""

    def __init__(self, vocab: int, d: int, d_ff: int, r: int, layers: int, seed: int = 0, mode: int = elas.ELAS_MODE_SPARSE24):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.vocab, self.d, self.layers, self.mode = vocab, d, layers, mode
        self.block_scale = (2 * layers) ** -0.5

        def normal(*shape, sigma=1.0):
            return torch.randn(shape, generator=gen, device="cuda") * sigma

        self.master = {"table": normal(vocab, d, sigma=d ** -0.5)}
        for k in range(layers):
            self.master[f"{k}.U_up"] = normal(d, r, sigma=d ** -0.5)
            self.master[f"{k}.V_up"] = normal(r, d_ff, sigma=r ** -0.5)
            self.master[f"{k}.U_down"] = normal(d_ff, r, sigma=d_ff ** -0.5)
            self.master[f"{k}.V_down"] = normal(r, d, sigma=r ** -0.5)
            self.master[f"{k}.gate"] = torch.full((d,), 0.5, device="cuda")
            self.master[f"{k}.w_post"] = torch.ones(d, device="cuda")
        for k in range(layers + 1):                      # the last one is the final norm
            self.master[f"{k}.w_pre"] = torch.ones(d, device="cuda")
        self.w = {k: v.to(BF) for k, v in self.master.items()}
        self.grad = {k: torch.empty_like(v) for k, v in self.master.items()}
        self.grads = elas.ElasTensors(self.grad.values())

    def factors(self, k: int):
        return [self.w[f"{k}.{n}"] for n in ("U_up", "V_up", "U_down", "V_down")]

    def around(self, k: int):
        """The operands of the norms around block k: after it, and before the next."""
        return dict(gate=self.w[f"{k}.gate"], w_post=self.w[f"{k}.w_post"], w_pre=self.w[f"{k + 1}.w_pre"],
                    block_scale=self.block_scale)

    def forward(self, ids: torch.Tensor):
        """The final norm's output and what the backward needs."""
        h = elas.elas_embed_fwd(ids, self.w["table"], self.d ** 0.5, dtype=torch.float32)
        n = elas.elas_norm_join_fwd(h, w_pre=self.w["0.w_pre"])["n"]
        kept = []
        for k in range(self.layers):
            ffn = elas.elas_lowrank_ffn_fwd(n, *self.factors(k), flags=self.mode)
            joined = elas.elas_norm_join_fwd(h, ffn["y"], **self.around(k))
            kept.append((n, ffn, joined["h"]))
            if k == 0:
                h0 = h
            h, n = joined["h"], joined["n"]
        return n, (ids, h0, kept)

    def backward(self, dn: torch.Tensor, saved) -> None:
        """Fills ``grad`` from the gradient of the final norm's output."""
        ids, h0, kept = saved
        dh = None
        for k in reversed(range(self.layers)):
            n, ffn, joined = kept[k]
            g = {"dh": torch.empty_like(joined), "db": torch.empty_like(n), "dgate": self.grad[f"{k}.gate"],
                 "dw_post": self.grad[f"{k}.w_post"], "dw_pre": self.grad[f"{k + 1}.w_pre"]}
            elas.elas_norm_join_bwd(dh, dn, joined, ffn["y"], **self.around(k), grads=g)
            f = {"dx": torch.empty_like(n), **{f"d{m}": self.grad[f"{k}.{m}"] for m in ("U_up", "V_up", "U_down", "V_down")}}
            elas.elas_lowrank_ffn_bwd(g["db"], n, *self.factors(k), ffn, flags=self.mode & elas.ELAS_MODE_DENSE, grads=f)
            dh, dn = g["dh"], f["dx"]
        g = {"dh": dh, "dw_pre": self.grad["0.w_pre"]}   # (in place)
        elas.elas_norm_join_bwd(dh, dn, h0, w_pre=self.w["0.w_pre"], grads=g)
        elas.elas_embed_bwd(ids, dh, self.vocab, self.d ** 0.5, dtable=self.grad["table"])

    def update(self, rate: float, max_norm: float) -> torch.Tensor:
        """Clips the gradients in place and takes a step; returns (norm, factor).
        Where the norm is not finite the factor is 0 and the step is skipped."""
        stats = elas.elas_grad_clip(self.grads, max_norm)
        step = torch.where(stats[1] > 0, -rate, 0.0)
        for k, m in self.master.items():
            m.add_(torch.nan_to_num(self.grad[k]) * step)
            self.w[k].copy_(m)
        return stats


def train(steps: int, tokens: int, layers: int, vocab: int = 1000, d: int = 256, d_ff: int = 688, r: int = 64, rate: float = 1.0,
          max_norm: float = 1.0, seed: int = 0, log=None) -> list:
    """Losses of the steps."""
    model = Stack(vocab, d, d_ff, r, layers, seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    follows = torch.randperm(vocab, generator=gen, device="cuda")
    targets = torch.randn(vocab, d, generator=gen, device="cuda")
    losses = []
    for step in range(steps):
        ids = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
        n, saved = model.forward(ids)
        diff = n.float() - targets[follows[ids]]
        model.backward((diff / tokens).to(BF), saved)
        stats = model.update(rate, max_norm)
        losses.append(diff.square().mean())
        if log and step % log == 0:
            print(f"step {step:4d}  loss {float(losses[-1]):.4f}  gradient norm {float(stats[0]):.3f}  factor {float(stats[1]):.3f}",
                  flush=True)
    return [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--layers", type=int, default=3)
    a = ap.parse_args()
    train(a.steps, a.tokens, a.layers, log=20)
