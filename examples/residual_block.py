"""A block on a residual stream, s = x + gate * norm(W2 gelu(W1 norm(x) + b1) + b2), trained with 8-bit operands: norms that write them, products with
their epilogue, gradients clipped by their common norm; and served with the same calls.

    python examples/residual_block.py [--rows 4096] [--width 2048] [--hidden 5504] [--steps 20]

What the backward pass needs of the forward pass: the 8-bit operands of both products, the activation's z, the second product's y and the stream x.
Weights, biases, norm weights and the gate stay in 32 bits; they are plain tensors, updated by plain steps against their clipped gradients.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2605_14929_amd as sop  # noqa: E402

NAMES = ("w1", "b1", "w2", "b2", "before", "after", "gate")


class ResidualBlock:
    """params: w1 [hidden, width], b1, w2 [width, hidden], b2, before [width] (norm in front), after [width] (norm behind), gate [width]; all float32."""

    def __init__(self, ctx, params):
        self.ctx, self.p = ctx, params
        self.refresh()

    def refresh(self):
        """8-bit operands of the weight matrices: blocks of 128 x 128, and the transposed codes that the input gradients read."""
        self.w1, self.w2 = (self.ctx.fp8_quantize(self.p[k], rows=128, transposed=True) for k in ("w1", "w2"))

    def forward(self, x, keep=True):
        c, p = self.ctx, self.p
        _, _, n8 = c.residual_norm(x, before=p["before"], fmt=sop.E4M3)
        h = c.fp8_linear(n8, self.w1, bias=p["b1"], act=sop.GELU, keep=keep)
        h, z = h if keep else (h, None)
        h8 = c.fp8_quantize(h)
        y = c.fp8_linear(h8, self.w2, bias=p["b2"])
        s, _, _ = c.residual_norm(x, y, after=p["after"], gate=p["gate"])
        if keep:
            self.kept = x, n8, z, h8, y
        return s

    def backward(self, ds):
        """(gradients by name, the stream's)"""
        c, p = self.ctx, self.p
        x, n8, z, h8, y = self.kept
        out = c.residual_norm_grad(ds, y=y, after=p["after"], gate=p["gate"], fmt=sop.E5M2)
        dw2, db2 = c.fp8_weight_grad(out.dy, h8), c.fp8_linear_grad(out.dy)[2]
        dz, dz8, db1 = c.fp8_linear_grad(c.fp8_matmul(out.dy8, self.w2, transposed=True), z, act=sop.GELU)
        dw1, dn = c.fp8_weight_grad(dz, n8), c.fp8_matmul(dz8, self.w1, transposed=True)
        front = c.residual_norm_grad(out.dr, dn, x, before=p["before"])
        return dict(zip(NAMES, (dw1, db1, dw2, db2, front.dbefore, out.dafter, out.dgate))), front.dr

    def step(self, grads, rate, most=1.0):
        """One step against the gradients, clipped to a common norm of `most`; their norm before that."""
        norm = self.ctx.clip_grads([grads[k] for k in NAMES], most)
        for k in NAMES:
            self.p[k].add_(grads[k], alpha=-rate)
        self.refresh()
        return norm


def make_params(width, hidden, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *z: torch.randn(z, generator=gen, device="cuda")  # noqa: E731
    return dict(w1=new(hidden, width) / width ** 0.5, b1=0.1 * new(hidden), w2=new(width, hidden) / hidden ** 0.5, b2=0.1 * new(width), before=1 + 0.1 * new(width),
                after=1 + 0.1 * new(width), gate=0.5 + 0.1 * new(width))


def plain(p, x):
    unit = lambda t: t * torch.rsqrt(t.square().mean(1, keepdim=True) + 1e-6)  # noqa: E731
    h = torch.nn.functional.gelu(unit(x) * p["before"] @ p["w1"].t() + p["b1"])
    return x + p["gate"] * p["after"] * unit(h @ p["w2"].t() + p["b2"])


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    a.add_argument("--rows", type=int, default=4096)
    a.add_argument("--width", type=int, default=2048)
    a.add_argument("--hidden", type=int, default=5504)
    a.add_argument("--steps", type=int, default=20)
    o = a.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((o.rows, o.width), generator=gen, device="cuda").bfloat16()
    wanted = plain(make_params(o.width, o.hidden, 3), x.float())
    block = ResidualBlock(sop.Context(0), make_params(o.width, o.hidden, 2))
    losses, norms = [], []
    for _ in range(o.steps):
        diff = block.forward(x).float() - wanted
        losses.append(float(diff.square().mean()))
        grads, _ = block.backward((diff * (2.0 / o.rows)).bfloat16())
        norms.append(float(block.step(grads, 0.1)))
    print(f"loss {losses[0]:.5f} -> {losses[-1]:.5f} after {o.steps} steps, norm of the gradients {norms[0]:.3f} -> {norms[-1]:.3f}")
    token = block.forward(x[:1].contiguous(), keep=False)
    exact = plain(block.p, x[:1].float())
    error = float((token.float() - exact).norm() / exact.norm())
    print(f"one token served, off by {error:.4f}")
    return losses, norms, error


if __name__ == "__main__":
    main()
