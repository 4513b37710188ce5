"""Recover the experts of a pruned layer and serve them in 8 bits.

    python examples/recover_experts.py [--steps 60]

A layer's experts are cut to a part of their channels (the keep table), trained back towards the unpruned layer's output
on random tokens, and then rounded to 8-bit integers:

  routing           the library's forward (routing copies: groups of rows per expert)
  forward           grouped products: gate and up limited in their rows, down in its columns
  backward          their input and weight gradients, the latter in bf16
  update            AdamW on fp32 master copies, states in 8 bits
  serving           the recovered experts as 8-bit products with a scale for each token and channel
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402


def silu(x):
    return x * torch.sigmoid(x)


class Experts:
    """Routed experts on grouped rows: products, gradients and update of one layer's pruned weights."""

    def __init__(self, weights, keep, max_rows, lr):
        E, I, d = weights[0].shape
        self.keep, self.lr = keep, lr
        self.w = [t.clone() for t in weights]  # gate, up [E, I, d], down [E, d, I]
        self.gate_up = fm.GroupedProduct(E, I, d, max_rows, keep_axis="N")
        self.down = fm.GroupedProduct(E, d, I, max_rows, keep_axis="K")
        self.opt = fm.AdamW(self.w, masters=[t.float() for t in self.w], state_bits=8, betas=(0.9, 0.95))
        self.dw = [torch.empty_like(t) for t in self.w]

    def forward(self, x, offsets):
        g = self.gate_up.forward(x, self.w[0], offsets, self.keep)
        u = self.gate_up.forward(x, self.w[1], offsets, self.keep)
        h = (silu(g.float()) * u.float()).bfloat16()
        return self.down.forward(h, self.w[2], offsets, self.keep), (x, g, u, h)

    def step(self, do, saved, offsets):
        """One update from the gradient of the experts' outputs."""
        x, g, u, h = saved
        dh = self.down.input_grad(do, self.w[2], offsets, self.keep).float()
        s, g, u = torch.sigmoid(g.float()), g.float(), u.float()
        dg = (dh * u * s * (1 + g * (1 - s))).bfloat16()
        du = (dh * g * s).bfloat16()
        self.gate_up.weight_grad(dg, x, offsets, self.keep, dw=self.dw[0])
        self.gate_up.weight_grad(du, x, offsets, self.keep, dw=self.dw[1])
        self.down.weight_grad(do, h, offsets, self.keep, dw=self.dw[2])
        self.opt.step(self.dw, self.lr)


class Int8Experts:
    """The same experts in 8-bit integers."""

    def __init__(self, weights, keep, max_rows):
        self.keep = keep
        self.gate = fm.Int8Product.from_weights(weights[0], max_rows, keep_axis="N")
        self.up = fm.Int8Product.from_weights(weights[1], max_rows, keep_axis="N")
        self.down = fm.Int8Product.from_weights(weights[2], max_rows, keep_axis="K")

    def forward(self, x, offsets):
        q, scale = fm.quantize_rows(x)
        g = self.gate.product(q, scale, offsets, self.keep)
        u = self.up.product(q, scale, offsets, self.keep)
        return self.down(u, offsets, self.keep, gate=g)  # silu(g) * u rounded in the same pass


def route(layer, x, logits):
    """(rows' tokens, rows' router weights, group offsets) of a batch, from the library's routing."""
    T, k, E = x.shape[0], layer.desc.top_k, layer.desc.E
    i32 = dict(dtype=torch.int32, device="cuda")
    r = dict(topk_w=torch.empty(T * k, dtype=torch.float32, device="cuda"), offsets=torch.empty(E + 1, **i32), perm=torch.empty(T * k, **i32))
    y = layer.forward(x, logits, dbg=r)
    a = r["perm"].long()  # every expert keeps some channels, so every assignment has its row
    return y, a // k, r["topk_w"][a], r["offsets"]


def combine(o, token, weight, T):
    return torch.zeros(T, o.shape[1], device="cuda").index_add_(0, token, o.float() * weight.unsqueeze(1))


def run(d=512, E=16, I=768, top_k=2, T=2048, kept=0.5, steps=60, lr=2e-3, seed=0):
    """Mean squared error against the unpruned layer before and after recovery, and in 8 bits; relative to its output."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return torch.empty(shape, device="cuda").normal_(0, std, generator=g).to(dtype)

    weights = [normal(E, I, d, std=d ** -0.5), normal(E, I, d, std=d ** -0.5), normal(E, d, I, std=I ** -0.5)]
    teacher = fm.Layer(d, E, I, top_k, max_tokens=T)
    teacher.set_weights(*weights)
    keep = torch.full((E,), int(kept * I), dtype=torch.int32, device="cuda")
    experts = Experts(weights, keep, T * top_k, lr)
    # a few batches of tokens that lie near a small number of directions, as hidden states do
    base = normal(64, d, dtype=torch.float32)
    batches = []
    for _ in range(4):
        x = (normal(T, 64, dtype=torch.float32) @ base / 8).bfloat16()
        batches.append((x, normal(T, E, dtype=torch.float32)))

    def error(model, x, logits):
        want, token, weight, offsets = route(teacher, x, logits)
        o = model.forward(x[token], offsets)
        y = combine(o[0] if isinstance(o, tuple) else o, token, weight, T)
        return float((y - want.float()).square().sum() / want.float().square().sum())

    before = error(experts, *batches[0])
    for s in range(steps):
        x, logits = batches[s % len(batches)]
        want, token, weight, offsets = route(teacher, x, logits)
        o, saved = experts.forward(x[token], offsets)
        dy = combine(o, token, weight, T) - want.float()
        experts.step((dy[token] * weight.unsqueeze(1)).bfloat16(), saved, offsets)
    after = error(experts, *batches[0])
    x, logits = batches[0]
    _, token, weight, offsets = route(teacher, x, logits)
    full = combine(experts.forward(x[token], offsets)[0], token, weight, T)
    served = combine(Int8Experts(experts.w, keep, T * top_k).forward(x[token], offsets), token, weight, T)
    rounding = float((served - full).norm() / full.norm())
    return before, after, rounding


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    b, a, r = run(steps=ap.parse_args().steps)
    print("error of the pruned layer %.3f, after recovery %.3f of the unpruned output's square; 8-bit serving differs by %.2f %%"
          % (b, a, 100 * r))
