"""The linear layer in 4 bits where blocks' powers of two are near the ends of their range: only what the sum itself is may overflow."""
import pytest
import torch

pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)
from paper_2608_24067_b200.layers import Layers  # noqa: E402


@pytest.fixture(scope="module")
def L():
    return Layers()


# powers of two of x and of the weights
POWERS = [(-60, 110), (-60, 117), (-60, 118), (-60, 121), (-60, 126), (-120, 127), (0, 119), (0, 121), (121, 0), (126, -60), (127, -120), (117, -60), (60, 60), (70, 70), (127, 127), (-100, -30), (-100, -39),
          (-39, -100), (-100, -100), (-126, -126)]


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 40, 5000])
@pytest.mark.parametrize("a,b", POWERS)
def test_powers_near_the_ends(L, T, a, b):
    """64 equal products of powers of two: exact in 4 bits and in fp32, and rounded once (to infinity or 0 where bf16 ends)."""
    D, F = 64, 264
    x = torch.full((T, D), 2.0 ** a, device="cuda", dtype=torch.bfloat16)
    w = torch.full((F, D), 2.0 ** b, device="cuda", dtype=torch.bfloat16)
    w[1] *= 1.5
    w[2, ::2] *= -1  # cancels
    w[3, :32] = 0.0
    y = L.linear_fp4(x, L.quantize_fp4(w))
    one = torch.full((F,), 64.0, dtype=torch.float64)
    one[1], one[2], one[3] = 96.0, 0.0, 32.0
    want = (one * 2.0 ** a * 2.0 ** b).float().bfloat16().cuda()
    assert torch.equal(y, want.expand(T, F)), (y[0, :5], want[:5])
    assert L.device_flags() == 0


@pytest.mark.parametrize("T", [1, 2, 4, 5])
def test_large_blocks_that_cancel(L, T):
    """Two blocks of 2^126 each that cancel, and a third that is left: no part of the sum is infinite."""
    x = torch.ones(T, 96, device="cuda", dtype=torch.bfloat16)
    w = torch.full((128, 96), 2.0 ** 122, device="cuda", dtype=torch.bfloat16)
    w[:, 32:64] *= -1
    w[:, 64:] = 2.0 ** 100
    y = L.linear_fp4(x, L.quantize_fp4(w))
    assert torch.equal(y, torch.full_like(y, 2.0 ** 105))
    gated = L.linear_fp4(x, L.quantize_fp4(torch.cat([w, torch.full_like(w, 2.0 ** -5)])), gated=True)
    assert torch.equal(gated, torch.full_like(gated, 3.0 * 2.0 ** 105))
