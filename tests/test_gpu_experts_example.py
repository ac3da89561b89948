"""The example that runs the map and the dense operators together: it learns, keeps its experts in use, and gives single tokens
what it gives them in a batch."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_experts_on_map():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import experts_on_map
    losses, counts, whole, single = experts_on_map.main(steps=40, n=2048, D=128, E=8, k=2, hidden=64)
    assert losses[-1] < 0.9 * losses[0]
    assert int(counts.min()) > 0
    # a batch rounds the hidden values to bf16 once more than single tokens do: a few roundings of 2^-8
    assert ((whole.float() - single.float()).abs() <= 2.0 ** -6 * whole.float().abs() + 2.0 ** -6).all()
