"""The dense operators' C entries without a GPU: null handles and arguments are refused before anything touches a device."""
import ctypes

import pytest
import torch

from paper_2608_24067_b200 import som


def test_null_handles():
    lib = som.load_library()
    assert lib.som_layers_create(None) == 1
    assert lib.som_layers_destroy(None) == 0
    assert lib.som_layers_last_cuda_error(None) == 0
    assert lib.som_layers_launch_count(None) == 0
    assert lib.som_layers_device_flags(None, None) == 1
    assert lib.som_linear(None, 2, 0, 0, 1, 8, 8, None, 8, None, None, None, 0, None, 8, None) == 1
    assert lib.som_linear_backward(None, 2, 0, 0, 1, 8, 8, None, 8, None, None, None, 8, None, None, None, None) == 1
    assert lib.som_route(None, 0, 0, 1, 4, 1, None, 4, None, 1, 1, 1, 1, 1.0, None, None, None, None) == 1
    assert lib.som_route_backward(None, 0, 0, 1, 4, 1, None, 4, None, None, 1, 1.0, None, None) == 1
    none = [None, 2, 0, 0, 1, 2, 1, 8, 8, None, 8, None, None, 0, None, None, None, None, None, 8]
    assert lib.som_experts(*none, None, 8, None) == 1
    assert lib.som_experts_backward(*none, None, None, None, None, None, None, None) == 1


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a machine without a GPU")
def test_no_device():
    lib = som.load_library()
    out = ctypes.c_void_p()
    assert lib.som_layers_create(ctypes.byref(out)) == 6 and not out.value
