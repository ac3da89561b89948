"""A block of dense layers behind a map, trained and then served in 4 bits.

The tokens of ``experts_on_map`` (a sample's two best units, projected) go through a block as a transformer has it behind its attention: the residual
stream is normed, a gated unit and a projection back are added to it, and it is normed once more.  The gradients come from the
``*_backward`` calls, ``AdamW`` moves fp32 masters and their bf16 copies, with moments in 8 bits.  For serving the two products' weights are
quantised to 4 bits once, and single tokens go through the same block.

    python examples/block_on_map.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from experts_on_map import tokens_of_map  # noqa: E402
from paper_2608_24067_b200.layers import AdamW, Layers  # noqa: E402

NAMES = ("norm_weight", "norm_bias", "up", "down", "last_weight", "last_bias")


class Block:
    def __init__(self, D, hidden, bits=8, seed=1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *s: torch.randn(*s, generator=gen, device="cuda") * s[-1] ** -0.5  # noqa: E731
        one, zero = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
        self.master = dict(zip(NAMES, (one, zero, new(2 * hidden, D), new(D, hidden), one.clone(), zero.clone())))
        self.w = {n: v.bfloat16() for n, v in self.master.items()}
        self.layers = Layers()
        self.optimizer = AdamW(self.layers, list(self.master.values()), copies=list(self.w.values()), bits=bits)
        self.served = None

    def forward(self, x):
        """Output, and what the gradient needs."""
        L, w = self.layers, self.w
        n = L.norm(x, w["norm_weight"], w["norm_bias"])
        h = L.linear(n, w["up"], act="silu", gated=True)
        last = L.norm(L.linear(h, w["down"]), w["last_weight"], w["last_bias"], residual=x)
        return last["y"], (x, n, h, last["sum"])

    def backward(self, kept, dy):
        """The gradients by name, and x's."""
        L, w = self.layers, self.w
        x, n, h, total = kept
        last = L.norm_backward(total, w["last_weight"], dy, w["last_bias"])
        down = L.linear_backward(h, w["down"], last["dx"])
        up = L.linear_backward(n, w["up"], down["dx"], act="silu", gated=True)
        first = L.norm_backward(x, w["norm_weight"], up["dx"], w["norm_bias"], dsum=last["dx"])
        return dict(zip(NAMES, (first["dweight"], first["dbias"], up["dweight"], down["dweight"], last["dweight"], last["dbias"]))), first["dx"]

    def step(self, x, target, rate=2e-3):
        y, kept = self.forward(x)
        error = y.float() - target.float()
        grads, _ = self.backward(kept, (2.0 / error.numel() * error * 256.0).bfloat16())  # (scaled up; AdamW's quotient does not see it)
        self.optimizer.step([grads[n] for n in NAMES], rate=rate, decay=0.01)
        return float(error.square().mean())

    def serve(self):
        """The products' weights as they are served."""
        self.served = {n: self.layers.quantize_fp4(self.w[n]) for n in ("up", "down")}

    def answer(self, x):
        """The block with the products' weights in 4 bits."""
        L, w = self.layers, self.w
        h = L.linear_fp4(L.norm(x, w["norm_weight"], w["norm_bias"]), self.served["up"], act="silu", gated=True)
        return L.norm(L.linear_fp4(h, self.served["down"]), w["last_weight"], w["last_bias"], residual=x)["y"]


def main(steps=40, n=4096, D=256, hidden=512):
    x, target = tokens_of_map(n=n, D=D)
    block = Block(D, hidden)
    losses = []
    for i in range(steps):
        losses.append(block.step(x, target))
        if i % 10 == 0 or i == steps - 1:
            print("step %3d  loss %.4f" % (i, losses[-1]))
    block.serve()
    whole, served = block.forward(x)[0], block.answer(x)
    off = float((served.float() - whole.float()).norm() / whole.float().norm())
    small = sum(q.codes.numel() + q.scales.numel() for q in block.served.values()) / sum(block.w[n].numel() * 2 for n in block.served)
    print("served in 4 bits: %.0f %% of the weights' bytes, outputs %.1f %% off" % (100 * small, 100 * off))
    single = torch.cat([block.answer(x[i:i + 1]) for i in range(8)])
    assert block.layers.device_flags() == 0
    return losses, off, served[:8], single


if __name__ == "__main__":
    main()
