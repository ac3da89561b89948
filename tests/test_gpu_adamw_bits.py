"""A step of AdamW with moments in 32 bits, bit by bit: parameters and their 16-bit copies are what the formula gives in fp32."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)
from paper_2608_24067_b200.layers import AdamW, Layers  # noqa: E402

F = np.float32


@pytest.fixture(scope="module")
def L():
    return Layers()


@pytest.mark.parametrize("param,copy", [("float32", "bfloat16"), ("float32", "float16"), ("float32", None), ("bfloat16", None), ("float16", None)])
@pytest.mark.parametrize("device_numbers", [False, True])
def test_every_operation_is_rounded_by_itself(L, param, copy, device_numbers):
    """numpy's fp32 rounds each product, sum, quotient and root to the nearest: no tolerance.  A product that is fused into the sum behind it moves a
    quarter of the fp32 parameters by one place."""
    n, rate, b1, b2, eps, decay, scale = 300001, 1e-2, 0.9, 0.999, 1e-8, 0.05, F(2.0 ** -7 * 1.3)
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
    p = (0.03 * new()).to(getattr(torch, param))
    c = None if copy is None else p.to(getattr(torch, copy))
    opt = AdamW(L, [p], None if c is None else [c])
    m, v = np.zeros(n, F), np.zeros(n, F)
    for t in (1, 2, 3):
        g = new() * torch.exp2(torch.randint(-12, 8, (n,), generator=gen, device="cuda").float())
        before = p.float().cpu().numpy()
        r = torch.tensor([rate], device="cuda") if device_numbers else rate
        opt.step([g], rate=r, beta1=b1, beta2=b2, eps=eps, decay=decay, step=torch.tensor([t], device="cuda") if device_numbers else t, scale=torch.tensor([scale], device="cuda"))
        x = g.cpu().numpy() * scale
        m = m * F(b1) + x * F(1 - b1)
        v = v * F(b2) + (x * x) * F(1 - b2)
        if device_numbers:
            rate = float(F(rate))  # (the rate as the device holds it)
        change = (m * F(1 / (1 - b1 ** t))) / (np.sqrt(v * F(1 / (1 - b2 ** t))) + F(eps))
        want = torch.from_numpy(before * F(1 - rate * decay) - change * F(rate)).cuda()
        got_m, got_v = (x[0].cpu().numpy() for x in opt.moments())
        assert np.array_equal(got_m, m) and np.array_equal(got_v, v)
        assert torch.equal(p, want.to(p.dtype)), "%d of %d" % (int((p != want.to(p.dtype)).sum()), n)
        if c is not None:
            assert torch.equal(c, want.to(c.dtype))
