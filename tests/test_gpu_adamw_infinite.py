"""AdamW with second moments that are infinite in fp32: they move nothing, in the step that makes them and in every one after it."""
import numpy as np
import pytest
import torch

import train_reference as ref

pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)
from paper_2608_24067_b200.layers import AdamW, Layers  # noqa: E402

HYPER = {"rate": 0.25, "beta1": 0.9, "beta2": 0.999, "decay": 0.01}


@pytest.fixture(scope="module")
def L():
    return Layers()


def host(t):
    return t.float().cpu().numpy().reshape(-1)


def check_step(opt, p, g, eps, t, step=None):
    """One step from the moments that `opt` holds, against the definition in 64 bits."""
    m, v = (host(x[0]) for x in opt.moments())
    before = host(p)
    opt.step([g], eps=eps, step=step, seed=t, **HYPER)
    m, v = ref.moments_step(m, v, host(g), HYPER["beta1"], HYPER["beta2"])
    want, tol = ref.param_step(before, m, v, HYPER["rate"], HYPER["beta1"], HYPER["beta2"], np.float64(np.float32(eps)), HYPER["decay"], t)
    rel, least = ref.half_step(p.dtype)
    off = np.abs(host(p).astype(np.float64) - want)
    assert (off <= tol + rel * np.abs(want) + least).all(), (t, int((~(off <= tol + rel * np.abs(want) + least)).sum()), host(p)[:8])
    return m, v


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-8, 1e-3, 1e-10])
@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("device_numbers", [False, True])
def test_an_infinite_second_moment_goes_on_moving_nothing(L, bits, eps, kind, device_numbers):
    """One gradient of 1e25 among ordinary ones, then ordinary gradients and none."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    p = torch.ones(1000, device="cuda").to(ref.TYPES[kind])
    opt = AdamW(L, [p], bits=bits)
    sign = torch.where(torch.rand(1000, generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    first = sign * (0.5 + torch.rand(1000, generator=gen, device="cuda"))
    first[300] = 1e25
    steps = [first, sign, torch.zeros_like(first), 1e-3 * sign]
    for t, g in enumerate(steps, start=1):
        check_step(opt, p, g, eps, t, torch.tensor([t], device="cuda") if device_numbers else None)
        after = p.double() if t == 1 else after
        v = opt.moments()[1][0]
        lost = torch.zeros(1000, dtype=torch.bool, device="cuda")
        lost[256:512] = bits == 8  # (in 8 bits the block's)
        lost[300] = True
        assert torch.equal(v.isinf(), lost) and not bool(v.isnan().any())
    # from then on what moves nothing decays alone: three roundings of values below 2 (an eps each at most) and, in fp32, three of the factor (an eps in all)
    keep = (1 - 0.25 * 0.01) ** 3
    assert bool(((p.double() - after * keep).abs() <= 4 * torch.finfo(p.dtype).eps)[lost].all())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-8, 1e-3, 1e-10])
def test_corrections_that_overflow(L, bits, eps):
    """Finite second moments up to the type's largest powers, whose correction by 1 / (1 - beta2) = 1000 is infinite or nearly so."""
    exponents = np.arange(235, 255)
    p = torch.ones(256 * len(exponents), device="cuda")
    opt = AdamW(L, [p], bits=bits)
    if bits == 8:
        code = torch.full((p.numel(),), 31 * 8 + 7, dtype=torch.uint8, device="cuda")  # 1.875 powers
        e = torch.from_numpy(exponents.astype(np.uint8)).cuda()
        m = torch.full_like(code, 8 * 15), torch.full_like(e, 127)  # 1
        opt.load([m], [(code, e)])
    else:
        opt.load([torch.ones_like(p)], [torch.from_numpy((1.875 * 2.0 ** (exponents - 127.0)).astype(np.float32)).cuda().repeat_interleave(256)])
    check_step(opt, p, torch.ones_like(p), eps, 1, step=1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("at", [0, 3, 5, 7])
def test_nan_beside_an_oversized_gradient(L, bits, at):
    """A NaN among the eight gradients that a thread takes is its element's alone."""
    p, g = torch.ones(256, device="cuda"), torch.ones(256, device="cuda")
    g[8:16] = 1e25
    g[8 + at] = float("nan")
    AdamW(L, [p], bits=bits).step([g], rate=0.25, decay=0.0)
    want = torch.full_like(p, 0.75)
    want[8:16] = 1.0
    keep = torch.arange(256, device="cuda") != 8 + at
    assert bool(p[8 + at].isnan()) and bool(((p[keep] - want[keep]).abs() <= 2.0 ** -20).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_that_was_left_out_is_counted(L, bits):
    """A scale that is not finite changes no tensor, but the number of the step goes on (the host does not learn of it); a caller who knows gives it."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    g, start = torch.randn(700, generator=gen, device="cuda"), torch.randn(700, generator=gen, device="cuda")
    bad = torch.tensor([float("inf")], device="cuda")

    def after(skipped, **kw):
        p = start.clone()
        opt = AdamW(L, [p], bits=bits)
        for _ in range(skipped):
            opt.step([g], scale=bad)
        opt.step([g], seed=5, **kw)
        return p, opt.steps

    plain, n = after(0)
    counted, n2 = after(1)
    given, n3 = after(1, step=1)
    second, _ = after(0, step=2)
    assert (n, n2, n3) == (1, 2, 1)
    assert torch.equal(given, plain) and torch.equal(counted, second) and not torch.equal(counted, plain)
