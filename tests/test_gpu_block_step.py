"""The block example's two ends: a step moves its masters and copies as AdamW's definition says, and what it serves is the block of its 4-bit
weights, each part against its definition in 64 bits."""
import os
import sys

import numpy as np
import pytest
import torch

import train_reference as ref
from test_gpu_norm import near

pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import block_on_map  # noqa: E402


def batch(T, D, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(T, D, generator=gen, device="cuda").bfloat16() for _ in range(2))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_moves_masters_and_copies(bits):
    T, D, hidden, rate = 200, 128, 64, 2e-3
    block = block_on_map.Block(D, hidden, bits=bits)
    x, target = batch(T, D, 3)
    for t in (1, 2):
        m, v = ([q.clone() for q in some] for some in block.optimizer.moments())  # (in 32 bits they are the moments themselves)
        before = {n: p.clone() for n, p in block.master.items()}
        y, kept = block.forward(x)
        error = y.float() - target.float()
        grads, _ = block.backward(kept, (2.0 / error.numel() * error * 256.0).bfloat16())
        block.step(x, target, rate=rate)
        for i, n in enumerate(block_on_map.NAMES):
            flat = [a.float().cpu().numpy().reshape(-1) for a in (before[n], m[i], v[i], grads[n], block.master[n])]
            mi, vi = ref.moments_step(flat[1], flat[2], flat[3], 0.9, 0.999)
            want, tol = ref.param_step(flat[0], mi, vi, rate, 0.9, 0.999, np.float64(np.float32(1e-8)), 0.01, t)
            assert (np.abs(flat[4] - want) <= tol + 2.0 ** -24 * np.abs(want)).all(), (t, n)
            assert (flat[4] != flat[0]).any()
            assert torch.equal(block.w[n], block.master[n].bfloat16())


@pytest.mark.parametrize("T", [1, 3, 70, 700])
def test_served_block_is_that_of_its_weights(T):
    D, hidden = 128, 256
    block = block_on_map.Block(D, hidden)
    x, target = batch(T, D, T)
    block.step(x, target)
    block.serve()
    L, w = block.layers, block.w
    assert all(torch.equal(L.quantize_fp4(w[n]).codes, block.served[n].codes) for n in ("up", "down"))
    values = {n: L.values_fp4(q, torch.float32) for n, q in block.served.items()}
    n = L.norm(x, w["norm_weight"], w["norm_bias"])
    h = L.linear_fp4(n, block.served["up"], act="silu", gated=True)
    near(h, *ref.fp4_linear(n, values["up"], None, None, "silu", True), "up")
    d = L.linear_fp4(h, block.served["down"])
    near(d, *ref.fp4_linear(h, values["down"], None, None, "none", False), "down")
    want, _, tol = ref.norm(d, w["last_weight"], w["last_bias"], x, 1e-5)
    near(block.answer(x), want, tol, "answer")
