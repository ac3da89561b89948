"""Experts behind a map: the library's dense operators run together on what a self-organizing map has learned.

Sparse binary samples are searched and the map is updated for a few epochs (``Som``).  Every sample then becomes a token: its
two best units' prototypes, projected to D numbers.  A layer of E experts learns to predict a vector that depends on the
sample's rarer features: the router's logits are a linear layer of the token, ``route`` picks k experts with a balance bias that is
moved by the counts it returns, ``experts`` adds the chosen experts' outputs to the token, and the three gradients train the
router and the experts by ``AdamW`` on fp32 master weights.  At the end single tokens go through the same layer, as in serving.

    python examples/experts_on_map.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_24067_b200 import synth  # noqa: E402
from paper_2608_24067_b200.layers import AdamW, Layers  # noqa: E402
from paper_2608_24067_b200.som import Som  # noqa: E402


def tokens_of_map(V=2000, side=16, n=4096, D=256, epochs=3, seed=0):
    """Token [n, D] and target [n, D] (bf16) of n samples from a small map."""
    M = side * side
    codebook = synth.fill_codebook(V, M, seed, device="cuda")
    batch = synth.sample_csr(n, V, 7.0, seed, device="cuda")
    som = Som(V, M, codebook)
    som.norms()
    for epoch in range(epochs):
        bmu, _ = som.bmu(batch.indptr, batch.indices)
        som.update(side, side, batch.indptr, batch.indices, bmu, radius=max(1, epochs - epoch))
        som.norms()
    bmu, _, second, _ = som.bmu2(batch.indptr, batch.indices)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    look = torch.randn(V, D, generator=gen, device="cuda") * V ** -0.5
    units = codebook.view(V, M).t() @ look  # [M, D]: prototypes, projected
    x = units[bmu.long()] + 0.5 * units[second.long()]
    x = (x - x.mean(0)) / x.std(0).clamp_min(1e-6)
    # the target: a fixed random vector for each feature, summed over the sample's, as far as the token does not show it
    row = torch.repeat_interleave(torch.arange(n, device="cuda"), (batch.indptr[1:] - batch.indptr[:-1]).long())
    sign = torch.randn(V, D, generator=gen, device="cuda")
    target = torch.zeros(n, D, device="cuda").index_add_(0, row, sign[batch.indices.long()])
    return x.bfloat16(), (x + 0.3 * target).bfloat16()


class ExpertLayer:
    """Router and experts with fp32 master weights; what the kernels see are bf16 copies."""

    def __init__(self, D, E, k, hidden, seed=1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *s, scale: torch.randn(*s, generator=gen, device="cuda") * scale  # noqa: E731
        self.master = {"router": new(E, D, scale=D ** -0.5), "w1": new(E, 2 * hidden, D, scale=D ** -0.5), "w2": new(E, D, hidden, scale=0.3 * hidden ** -0.5),
                       "b1": torch.zeros(E, 2 * hidden, device="cuda"), "b2": torch.zeros(E, D, device="cuda")}
        self.w = {n: v.bfloat16() for n, v in self.master.items()}
        self.balance = torch.zeros(E, device="cuda")
        self.k = k
        self.layers = Layers()
        self.optimizer = AdamW(self.layers, list(self.master.values()), copies=list(self.w.values()))

    def forward(self, x):
        logits = self.layers.linear(x, self.w["router"])
        routed = self.layers.route(logits, self.k, score="sigmoid", bias=self.balance, renorm=True)
        y = self.layers.experts(x, routed["indices"], routed["weights"], self.w["w1"], self.w["w2"], self.w["b1"], self.w["b2"], residual=x)
        return y, logits, routed

    def step(self, x, target, rate=3e-3, balance_rate=0.01):
        y, logits, routed = self.forward(x)
        error = y.float() - target.float()
        dy = (2.0 / error.numel() * error * 256.0).bfloat16()  # scaled up: bf16 keeps the same precision, the sums stay comfortable
        g = self.layers.experts_backward(x, routed["indices"], routed["weights"], self.w["w1"], self.w["w2"], dy, self.w["b1"], self.w["b2"])
        dlogits = self.layers.route_backward(logits, routed["indices"], g["dweights"], score="sigmoid", renorm=True)
        g["drouter"] = self.layers.linear_backward(x, self.w["router"], dlogits)["dweight"]
        self.optimizer.step([g["d" + n] for n in self.master], rate=rate, beta2=0.99, decay=0.0)
        # an expert that gets fewer tokens than its share becomes easier to choose (the choice alone; the weights do not see it)
        counts = routed["counts"].float()
        self.balance += balance_rate * torch.sign(counts.mean() - counts)
        return float(error.square().mean()), routed["counts"]


def main(steps=60, n=4096, D=256, E=16, k=4, hidden=128):
    x, target = tokens_of_map(n=n, D=D)
    layer = ExpertLayer(D, E, k, hidden)
    losses = []
    for i in range(steps):
        loss, counts = layer.step(x, target)
        losses.append(loss)
        if i % 10 == 0 or i == steps - 1:
            print("step %3d  loss %.4f  tokens of an expert: least %d, most %d" % (i, loss, int(counts.min()), int(counts.max())))
    whole, _, _ = layer.forward(x)
    single = torch.cat([layer.forward(x[i:i + 1])[0] for i in range(8)])
    assert layer.layers.device_flags() == 0
    return losses, counts, whole[:8], single


if __name__ == "__main__":
    main()
