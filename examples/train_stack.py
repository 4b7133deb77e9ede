"""Trains a small stack of ELAS blocks with the operators around them, as a
training step uses them together:

    ids -> embedding -> [norm -> low-rank 2:4 FFN -> norm, gate, residual sum] x L
        -> norm -> logits -> token loss -> the same backward -> gradient norm -> AdamW

    python examples/train_stack.py [--steps N] [--tokens T] [--layers L] [--bits 8]

Each token learns to predict the token that follows it (a permutation of the
vocabulary), so no sequence mixing is needed.  torch provides the memory and the
dense products of the logits' layer; everything else is libelas: the loss writes its
gradient over the logits, and the update of the float32 master weights clips the
gradients and writes the bf16 copies.
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
    """Weights of the stack: float32 masters, their bf16 copies and gradients, and AdamW's state.  The logits' layer is
    apart from the rest: ``forward`` and ``backward`` go to and from the final norm's output."""

    def __init__(self, vocab: int, d: int, d_ff: int, r: int, layers: int, seed: int = 0, mode: int = elas.ELAS_MODE_SPARSE24, bits: int = 32):
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
        self.head_master = normal(vocab, d, sigma=d ** -0.5)
        self.head = self.head_master.to(BF)
        self.head_grad = torch.empty_like(self.head_master)
        self.grads = elas.ElasTensors([*self.grad.values(), self.head_grad])
        masters = [*self.master.values(), self.head_master]
        self.opt = elas.ElasAdamW(masters, copies=[*self.w.values(), self.head], decay=[0.1 * (m.dim() > 1) for m in masters], bits=bits)

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

    def loss(self, n: torch.Tensor, targets: torch.Tensor):
        """The mean cross-entropy of the targets ([1], with its z term beside it: stats [2]), the gradient of n;
        fills ``head_grad``."""
        logits = n @ self.head.t()
        out = {"stats": torch.empty(2, device="cuda"), "dlogits": logits}      # (the gradient over the logits)
        elas.elas_token_loss(logits, targets, reduce=1 / targets.numel(), z_coef=1e-4, out=out)
        self.head_grad.copy_(logits.t() @ n)
        return out["stats"], logits @ self.head

    def update(self, rate: float, max_norm: float) -> torch.Tensor:
        """A step of AdamW with the gradients clipped to max_norm; returns their norm.  Where it is not
        finite the step is skipped."""
        norm = elas.elas_grad_norm(self.grads)
        elas.elas_adamw_step(self.opt, self.grads, rate, beta2=0.95, norm=norm, max_norm=max_norm)
        return norm


def train(steps: int, tokens: int, layers: int, vocab: int = 1000, d: int = 256, d_ff: int = 688, r: int = 64, rate: float = 1e-2,
          max_norm: float = 1.0, seed: int = 0, bits: int = 32, log=None) -> list:
    """Losses of the steps."""
    model = Stack(vocab, d, d_ff, r, layers, seed, bits=bits)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    follows = torch.randperm(vocab, generator=gen, device="cuda")
    losses = []
    for step in range(steps):
        ids = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
        n, saved = model.forward(ids)
        stats, dn = model.loss(n, follows[ids])
        model.backward(dn, saved)
        norm = model.update(rate, max_norm)
        losses.append(stats[0])
        if log and step % log == 0:
            print(f"step {step:4d}  loss {float(stats[0]):.4f}  gradient norm {float(norm):.3f}", flush=True)
    return [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--layers", type=int, default=3)
    ap.add_argument("--bits", type=int, choices=(8, 32), default=32, help="of AdamW's moments")
    a = ap.parse_args()
    train(a.steps, a.tokens, a.layers, bits=a.bits, log=20)
