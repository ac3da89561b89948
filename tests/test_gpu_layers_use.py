"""GPU tests of how the dense operators are used: other streams."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_24067_b200 import layers
    return layers.Layers()


def _normal(gen, *shape, scale=1.0, dtype=FP32):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype).cuda()


def test_memory_of_another_stream(L):
    """Outputs on another stream do not take memory that the current stream has still to write; what either stream still reads is not
    handed out again."""
    gen = torch.Generator().manual_seed(1)
    x, w = _normal(gen, 100, 256, dtype=BF16), _normal(gen, 512, 256, dtype=BF16)
    want = L.linear(x, w, act="gelu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    # the current stream still has to write memory that was freed
    torch.cuda._sleep(50000000)
    late = torch.empty_like(want).fill_(7.0)
    at = late.data_ptr()
    del late
    got = L.linear(x, w, act="gelu", stream=side)
    assert got.data_ptr() != at
    side.synchronize()
    assert torch.equal(got, want)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    # an input given up while the other stream has still to read it
    copy = x.clone()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(50000000)
    got = L.linear(copy, w, act="gelu", stream=side)
    at = copy.data_ptr()
    del copy
    other = torch.empty_like(x).fill_(math.nan)
    assert other.data_ptr() != at
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    # an output given up while the current stream has still to read it
    torch.cuda._sleep(50000000)
    read = got.clone()
    at = got.data_ptr()
    del got
    again = L.linear(-x, w, act="gelu", stream=side)
    assert again.data_ptr() != at
    torch.cuda.synchronize()
    assert torch.equal(read, want)
