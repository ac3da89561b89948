"""Norm, AdamW and matrices in 4 bits without a GPU: null handles and bad arguments are refused before anything touches a device."""
import ctypes

import numpy as np
import pytest
import torch

import train_reference as ref
from paper_2608_24067_b200 import layers, som
from test_layers_cpu import BF16, _handle, _On, _Refused

U8, F32 = torch.uint8, torch.float32


def test_null_handles():
    lib = som.load_library()
    assert lib.som_norm(None, 2, 1, 8, None, 8, None, None, 2, None, 0, 1e-5, None, 0, None, 8, None) == 1
    assert lib.som_norm_backward(None, 2, 1, 8, None, 8, None, 2, None, 8, None, 0, 1e-5, None, None, None, None) == 1
    assert lib.som_adamw(None, 0, 0, -1, 32, 0, None, None, None) == 1
    assert lib.som_adamw_moments(None, 0, None, None, None, None) == 1
    assert lib.som_fp4_quantize(None, 2, 1, 32, None, 32, None, None, None) == 1
    assert lib.som_fp4_values(None, 2, 1, 32, None, None, None, 32, None) == 1
    assert lib.som_fp4_linear(None, 2, 0, 0, 1, 32, 8, None, 32, None, None, None, None, 0, None, 8, None) == 1


def test_scale_bytes():
    size = som.load_library().som_fp4_scale_bytes
    assert size(0, 32) == 0 and size(1, 32) == 1024 and size(128, 256) == 1024 and size(129, 288) == 4096
    for rows, D in ((1, 0), (1, 31), (1, 40), (-1, 32), (1 << 30, 32), (1, (1 << 24) + 32)):
        assert size(rows, D) == -1
    # the order in memory holds every byte once
    rows, blocks = np.arange(300)[:, None], np.arange(2080 // 32)[None]
    at = ref.scale_at(rows, blocks, 2080)
    assert len(np.unique(at)) == at.size and at.max() < size(300, 2080)


def test_structures_are_the_library_s():
    assert ctypes.sizeof(layers._Tensor) == 64 and ctypes.sizeof(layers._Step) == 80


T, D = 4, 64
TENSORS = {
    "norm": {"x": ((T, D), BF16), "weight": ((D,), F32), "bias": ((D,), F32), "residual": ((T, D), BF16), "out": ((T, D), BF16)},
    "norm_backward": {"x": ((T, D), BF16), "weight": ((D,), BF16), "dy": ((T, D), BF16), "bias": ((D,), BF16), "dsum": ((T, D), BF16)},
    "quantize_fp4": {"x": ((T, D), BF16)},
    "values_fp4": {"codes": ((T, D // 2), U8), "scales": ((1024,), U8)},
    "linear_fp4": {"x": ((T, D), BF16), "codes": ((32, D // 2), U8), "scales": ((1024,), U8), "bias": ((32,), BF16), "residual": ((T, 32), BF16), "out": ((T, 32), BF16)},
}


def _call(name, elsewhere=None, where=1):
    args = {n: torch.zeros(shape, dtype=dtype).as_subclass(_On) for n, (shape, dtype) in TENSORS[name].items()}
    if elsewhere:
        shape, dtype = TENSORS[name][elsewhere]
        args[elsewhere] = torch.zeros(shape, dtype=dtype)  # where < 0: on the host
        if where >= 0:
            args[elsewhere] = args[elsewhere].as_subclass(type("_Other", (_On,), {"index": where}))
    if "codes" in args:
        args["q" if name == "values_fp4" else "weight"] = layers.Fp4Matrix(args.pop("codes"), args.pop("scales"))
    h = _handle()
    fake = type(h._lib)()
    fake.som_fp4_scale_bytes = som.load_library().som_fp4_scale_bytes  # (sizes alone)
    h._lib = fake
    return getattr(h, name)(**args)


@pytest.mark.parametrize("name", TENSORS)
def test_tensors_of_another_device_are_refused(name):
    with pytest.raises(_Refused):  # all on the handle's device: the call goes through to the library
        _call(name)
    for n in TENSORS[name]:
        with pytest.raises(ValueError):
            _call(name, n, 1)
        with pytest.raises((TypeError, ValueError)):
            _call(name, n, -1)


def _on(*shape, t=F32, index=0):
    return torch.zeros(*shape, dtype=t).as_subclass(_On if index == 0 else type("_Other", (_On,), {"index": index}))


def test_optimiser_refuses_before_it_changes_anything():
    h = _handle()
    p, q, g = _on(10), _on(3, 4, t=BF16), _on(10)
    for bad in (lambda: layers.AdamW(h, [p, q, p]), lambda: layers.AdamW(h, [p, p[3:]]), lambda: layers.AdamW(h, [torch.zeros(3)]), lambda: layers.AdamW(h, [_on(3, index=1)]),
                lambda: layers.AdamW(h, [q.t()]), lambda: layers.AdamW(h, [p], copies=[p[:10].view(10)]), lambda: layers.AdamW(h, [q], copies=[q]), lambda: layers.AdamW(h, [p], bits=4)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    opt = layers.AdamW(h, [p, q], bits=8)
    with pytest.raises(_Refused):
        opt.step([g, _on(3, 4, t=BF16)])
    for bad in ([g], [g, _on(3, 4, t=torch.float16)], [g, _on(12, t=BF16)], [g, _on(3, 4, t=BF16, index=1)], [torch.zeros(10), _on(3, 4, t=BF16)]):
        with pytest.raises((TypeError, ValueError)):
            opt.step(bad)
    assert opt.steps == 0


def test_reference_codes():
    """The reference's own encoding: exact values keep, others become one of their neighbours, up as often as the random bits say."""
    rng = np.random.default_rng(0)
    for signed in (True, False):
        code = rng.integers(0, 256, 4096).astype(np.uint8)
        if signed:
            code[code == 128] = 0
        code[0::256] = 120 if signed else 248  # each block's largest: the exponent is its own
        code[code > (246 if not signed else 255)] = 248
        if signed:
            code = np.where((code & 127) > 120, 120, code).astype(np.uint8)
        e = rng.integers(60, 180, 16).astype(np.uint8)
        x = ref.decode(code, e, signed).astype(np.float32)
        for bits in (0, 0xFFFFFFFF):
            again, e2 = ref.encode(x, signed, np.full(4096, bits, np.uint32))
            assert np.array_equal(e, e2) and np.array_equal(ref.decode(again, e2, signed), x)
        y = (x * np.float32(1.01)).astype(np.float32)
        low, e0 = ref.encode(y, signed, np.zeros(4096, np.uint32))
        high, e1 = ref.encode(y, signed, np.full(4096, 0xFFFFFFFF, np.uint32))
        assert np.array_equal(e0, e1)
        lo, hi = np.abs(ref.decode(low, e0, signed)), np.abs(ref.decode(high, e1, signed))
        assert (lo <= np.abs(y)).all() and (hi >= np.abs(y) * (1 - 2.0 ** -15)).all() and ((high.astype(int) - low) <= 1).all()
