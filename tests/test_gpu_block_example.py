"""The example that trains a block (norm, gated unit, projection, AdamW) and serves it in 4 bits: it runs, its gradients are those of the
formula, and single tokens get what they get in a batch."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import block_on_map  # noqa: E402


def test_block_on_map():
    losses, off, served, single = block_on_map.main(steps=6, n=1024, D=128, hidden=256)
    assert all(v == v and v < float("inf") for v in losses) and off == off
    # the same sums in another order, rounded to bf16: hidden values that fall on the other side of a rounding (2^-8 of a value) may take
    # another 4-bit value (up to a sixth of it) in the second product: 1 of 256 of them, spread over sums of 256
    assert float((served.float() - single.float()).abs().max()) <= 2.0 ** -3
    assert float((served.float() - single.float()).norm()) <= 2.0 ** -6 * float(served.float().norm())


@pytest.mark.parametrize("T,D,hidden", [(1, 64, 32), (77, 256, 384), (1000, 512, 128)])
def test_gradients(T, D, hidden):
    """The chained calls against autograd in 64 bits on the same bf16 weights.  Every product reads operands rounded to bf16 (2^-8 of a value each):
    over the chain of two products and two norms four to six such roundings, independent of each other, 2^-8 / sqrt(3) in the norm each."""
    block = block_on_map.Block(D, hidden)
    gen = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, D, generator=gen, device="cuda").bfloat16()
    dy = torch.randn(T, D, generator=gen, device="cuda").bfloat16()
    for n in ("norm_weight", "last_weight"):
        block.w[n].add_(0.2 * torch.randn(D, generator=gen, device="cuda").bfloat16())
    y, kept = block.forward(x)
    grads, dx = block.backward(kept, dy)
    w = {n: v.double().requires_grad_() for n, v in block.w.items()}
    x64 = x.double().requires_grad_()
    h = torch.nn.functional.layer_norm(x64, (D,), w["norm_weight"], w["norm_bias"]) @ w["up"].t()
    h = torch.nn.functional.silu(h[:, :hidden]) * h[:, hidden:]
    want = torch.nn.functional.layer_norm(h @ w["down"].t() + x64, (D,), w["last_weight"], w["last_bias"])
    want.backward(dy.double())
    far = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    allowed = 2 * 6 ** 0.5 * 2.0 ** -8  # (six of them, and as much again for what the norms' divisions do with them)
    assert far(y, want.detach()) < allowed and far(dx, x64.grad) < allowed
    for n in block_on_map.NAMES:
        assert far(grads[n], w[n].grad) < allowed, n
