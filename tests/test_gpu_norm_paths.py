"""The forms of the norm and its gradient that longer and odd rows take, and the columns' sums of many rows."""
import numpy as np
import pytest
import torch

import train_reference as ref
from test_gpu_norm import check, inputs

pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)
from paper_2608_24067_b200.layers import Layers  # noqa: E402


@pytest.fixture(scope="module")
def L():
    return Layers()


# rows beyond the registers with several parts of the rows, on 16 bytes and not; rows off 16 bytes of 256 and 512 threads
SIZES = [(1000, 8200), (700, 9001), (300, 20001), (70, 40000), (40, 4095), (20, 8001), (150, 2049), (33, 6000), (9, 16384), (5, 16385)]


@pytest.mark.parametrize("kind", ref.TYPES)
@pytest.mark.parametrize("T,D", SIZES)
def test_sizes(L, T, D, kind):
    check(L, *inputs(T, D, kind, seed=T + D))


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("T,D,apart,shift", [(300, 8200, 8, 0), (300, 8200, 0, 1), (200, 9000, 3, 5), (64, 4096, 0, 3), (64, 8192, 5, 0)])
def test_fp32_weights_and_strides(L, T, D, apart, shift, kind):
    check(L, *inputs(T, D, kind, weights="fp32", apart=apart, shift=shift, seed=D))


def test_columns_of_many_rows_are_summed_in_short_chains(L):
    """Terms chosen so that a sum of 4096 of them one after the other (every eighth row of a half) is cut by nearly half a step at each: what a sum loses
    is bounded by its longest chain, a 64th of the rows."""
    T, D = 65536, 8200
    total, terms = np.float32(0), []
    for _ in range(T // 16):
        half = np.spacing(total) / 2 if total > 2 else np.float32(0)
        d = np.float32(1.0) + np.float32(half * (1 - 2.0 ** -3)) if half else np.float32(1.0)
        terms.append(d)
        total = np.float32(total + d)
    terms = torch.from_numpy(np.array(terms, np.float32)).cuda()
    dy = terms[torch.arange(T, device="cuda") % (T // 2) // 8][:, None].expand(T, D).contiguous()
    x = torch.zeros(T, D, device="cuda")
    x[:, ::2] = 1.0
    got = L.norm_backward(x, torch.ones(D, device="cuda"), dy, torch.zeros(D, device="cuda"))["dbias"]
    want = dy[:, 0].double().sum()
    off = float((got.double() - want).abs().max() / want / ref.U)
    assert off <= ref.chain(T) + 4, off
