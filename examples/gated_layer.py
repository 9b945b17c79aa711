"""A gated layer, y = (silu(x Wg^T) * (x Wu^T)) Wd^T, trained with 8-bit operands and activations kept in 8 bits, then searched, packed and
served from its packed codes.

    python examples/gated_layer.py [--rows 4096] [--width 2048] [--hidden 5504] [--steps 20]

Training: every operand of a product is 8-bit floats under one power-of-two scale for each block of 128; what the backward pass needs of the
forward pass is those operands themselves (x, h) and the 8-bit checkpoints of the gated unit.  The master weights stay in 32 bits.
Serving: each weight matrix becomes 4-bit codes of a pair of codebooks under 8-bit block scales (sop_search_layer), and the products read those.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2605_14929_amd as sop  # noqa: E402
from paper_2605_14929_amd.layer_search import search_layer  # noqa: E402


class GatedLayer:
    """Master weights gate, up [hidden, width] and down [width, hidden] in 32 bits, their 8-bit operands, and one pass's checkpoints."""

    def __init__(self, ctx, gate, up, down):
        self.ctx, self.weights = ctx, [gate, up, down]
        self.refresh()

    def refresh(self):
        """8-bit operands of the master weights: blocks of 128 x 128, and the transposed codes that the input gradients read."""
        self.gate, self.up, self.down = (self.ctx.fp8_quantize(w, rows=128, transposed=True) for w in self.weights)

    def forward(self, x):
        c = self.ctx
        x8 = c.fp8_quantize(x)
        h8, gate8, up8 = c.fp8_gated(c.fp8_matmul(x8, self.gate), c.fp8_matmul(x8, self.up))
        self.kept = x8, h8, gate8, up8
        return c.fp8_matmul(h8, self.down)

    def kept_bytes(self):
        return sum(q.codes.numel() + q.scales.numel() for q in self.kept)

    def backward(self, dy):
        """(gradients of gate, up, down in 32 bits, of x in bf16)."""
        c = self.ctx
        x8, h8, gate8, up8 = self.kept
        dh = c.fp8_matmul(c.fp8_quantize(dy, fmt=sop.E5M2), self.down, transposed=True)
        ddown = c.fp8_weight_grad(dy, h8)
        dgate, dup, dgate8, dup8 = c.fp8_gated_grad(gate8, up8, dh)
        dx = c.fp8_matmul(dgate8, self.gate, transposed=True) + c.fp8_matmul(dup8, self.up, transposed=True)
        return [c.fp8_weight_grad(dgate, x8), c.fp8_weight_grad(dup, x8), ddown], dx

    def step(self, grads, rate):
        for w, g in zip(self.weights, grads):
            w.add_(g, alpha=-rate)
        self.refresh()


class PackedLayer:
    """The same layer from packed codes: a search over pairs of codebooks for each matrix, blocks of 16 along the rows."""

    def __init__(self, ctx, weights, x):
        self.ctx = ctx
        fmt, atoms = sop.fmt_by_name("UE4M3"), sop.build_alphabet(["NF4", "SH4"])
        gate, up, down = weights
        norms = x.float().square().mean(0).sqrt()                       # of each matrix's input, channel by channel
        hidden = torch.nn.functional.silu(x.float() @ gate.t()) * (x.float() @ up.t())
        self.layers = []
        for w, c in ((gate, norms), (up, norms), (down, hidden.square().mean(0).sqrt())):
            shift = max(0, int(torch.floor(torch.log2(1.0 / w.abs().max()))))   # the scales of weights this small lie in the format's range
            r = search_layer(ctx, w, c, 16, fmt, atoms, p_grid=(), k=shift, pack=True)
            self.layers.append(sop.PackedWeights(r.words, r.payload, *w.shape, 16, r.n_bits, fmt, [r.table_a, r.table_b], k=shift))

    def bytes(self):
        return sum(p.words.numel() * 2 + p.payload.numel() for p in self.layers)

    def forward(self, x):
        gate, up, down = self.layers
        g, u = self.ctx.packed_matmul(x, gate), self.ctx.packed_matmul(x, up)
        return self.ctx.packed_matmul(torch.nn.functional.silu(g) * u, down)


def make_weights(width, hidden, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda n, k: torch.randn((n, k), generator=gen, device="cuda") / k ** 0.5  # noqa: E731
    return [new(hidden, width), new(hidden, width), new(width, hidden)]


def plain(weights, x):
    gate, up, down = weights
    return (torch.nn.functional.silu(x @ gate.t()) * (x @ up.t())) @ down.t()


def off(a, b):
    return float((a.detach().float() - b.detach().float()).norm() / b.detach().float().norm())


def timed(f, n=20):
    f()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(n):
        f()
    torch.cuda.synchronize()
    return (time.perf_counter() - t) / n * 1e6


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    a.add_argument("--rows", type=int, default=4096)
    a.add_argument("--width", type=int, default=2048)
    a.add_argument("--hidden", type=int, default=5504)
    a.add_argument("--steps", type=int, default=20)
    o = a.parse_args(argv)
    ctx = sop.Context(0)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((o.rows, o.width), generator=gen, device="cuda").bfloat16()
    start = make_weights(o.width, o.hidden, 2)
    wanted = plain([w + 0.1 * d for w, d in zip(start, make_weights(o.width, o.hidden, 3))], x.float())
    layer = GatedLayer(ctx, *(w.clone() for w in start))
    losses, kept = [], 0
    for _ in range(o.steps):
        y = layer.forward(x)
        kept = layer.kept_bytes()
        diff = y.float() - wanted
        losses.append(float(diff.square().mean()))
        grads, _ = layer.backward((diff * (2.0 / o.rows)).bfloat16())
        layer.step(grads, 0.1)
    wide = 2 * o.rows * (o.width + 3 * o.hidden)
    print(f"loss {losses[0]:.5f} -> {losses[-1]:.5f} after {len(losses)} steps; kept for the backward pass {kept / 2**20:.1f} MiB, in bf16 {wide / 2**20:.1f} MiB")
    y = layer.forward(x)
    dy = (y.float() - wanted).bfloat16()
    exact = plain(layer.weights, x.float())
    print(f"8-bit output off by {off(y, exact):.4f}; forward {timed(lambda: layer.forward(x)):.0f} us, backward {timed(lambda: layer.backward(dy)):.0f} us")
    packed = PackedLayer(ctx, layer.weights, x)
    token = x[:1].contiguous()
    error = off(packed.forward(x), exact)
    print(f"packed output off by {error:.4f}, {packed.bytes() * 8 / sum(w.numel() for w in layer.weights):.2f} bits a weight; "
          f"one token {timed(lambda: packed.forward(token)):.0f} us, {o.rows} rows {timed(lambda: packed.forward(x)):.0f} us")
    return losses, off(y, exact), error


if __name__ == "__main__":
    main()
