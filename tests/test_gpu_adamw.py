"""A step of AdamW over many tensors against its definition: moments bit by bit, parameters in 64 bits."""
import itertools

import numpy as np
import pytest
import torch

import train_reference as ref
from train_reference import TYPES, U

pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)
from paper_2608_24067_b200.layers import AdamW, Layers  # noqa: E402
from paper_2608_24067_b200.som import SomError  # noqa: E402


@pytest.fixture(scope="module")
def L():
    return Layers()


ODD = [(1,), (7,), (256,), (257,), (2048,), (33, 67), (3, 5, 700), (0,), (4099,)]


def tensors(shapes, param, grad, copy=None, seed=0, shift=0, steps=3):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def new(shape, t, scale):
        v = (torch.randn(shape, generator=gen, device="cuda") * scale).to(t)
        if not shift:
            return v
        whole = torch.zeros(v.numel() + shift, device="cuda", dtype=t)
        return whole[shift:].view(shape).copy_(v)

    params = [new(s, TYPES[param], 1.0) for s in shapes]
    # sizes over many powers of two in one tensor, zeros among them
    grads = [[(new(s, TYPES[grad], 1.0) * torch.exp2(torch.randint(-20, 1, s, generator=gen, device="cuda").float()) * (torch.rand(s, generator=gen, device="cuda") > 0.1)).to(TYPES[grad])
              for s in shapes] for _ in range(steps)]
    if shift:
        grads = [[new(g.shape, g.dtype, 0.0).copy_(g) for g in some] for some in grads]
    copies = [new(s, TYPES[copy], 1.0) for s in shapes] if copy else None
    return params, grads, copies


def host(t):
    return t.detach().float().cpu().numpy().reshape(-1)


def check_steps(opt, params, grads, copies, kinds, scale=None, **kw):
    hyper = {"rate": 1e-2, "beta1": 0.9, "beta2": 0.99, "eps": 1e-8, "decay": 0.1, **kw}
    m, v = ([np.zeros(p.numel(), np.float32) for p in params] for _ in range(2))
    for k, some in enumerate(grads):
        before = [host(p) for p in params]
        opt.step(some, scale=scale, seed=11 + k, **hyper)
        got_m, got_v = opt.moments()
        codes = opt.state() if opt.bits == 8 else None
        for i, p in enumerate(params):
            g = host(some[i])
            if scale is not None:
                g = g * np.float32(float(scale))
            m[i], v[i] = ref.moments_step(m[i], v[i], g, hyper["beta1"], hyper["beta2"])
            want, tol = ref.param_step(before[i], m[i], v[i], hyper["rate"], hyper["beta1"], hyper["beta2"], hyper["eps"], hyper["decay"], k + 1)
            rel, least = ref.half_step(p.dtype)
            off = np.abs(host(p).astype(np.float64) - want)
            assert (off <= tol + rel * np.abs(want) + least).all(), (kinds, k, p.shape, (off / (tol + rel * np.abs(want) + least)).max())
            if copies:
                if params[i].dtype is torch.float32:
                    assert torch.equal(copies[i], p.to(copies[i].dtype))
            if opt.bits == 8 and p.numel():
                r = ref.random_bits(p.numel(), 11 + k, i)
                for which, (mine, signed) in enumerate(((m, True), (v, False))):
                    code, e = ref.encode(mine[i], signed, r)
                    got_code, got_e = codes[which][i]
                    assert np.array_equal(got_e.cpu().numpy(), e), (kinds, k, p.shape, signed)
                    assert np.array_equal(got_code.cpu().numpy().reshape(-1), code), (kinds, k, p.shape, signed)
                    mine[i] = ref.decode(code, e, signed).astype(np.float32)
            assert np.array_equal(host(got_m[i]), m[i]) and np.array_equal(host(got_v[i]), v[i]), (kinds, k, p.shape)


KINDS = [("fp32", "fp32", None), ("fp32", "bf16", "bf16"), ("fp32", "fp16", "fp16"), ("fp32", "bf16", None), ("fp32", "fp32", "bf16"), ("bf16", "bf16", None), ("bf16", "fp32", None),
         ("fp16", "fp16", None), ("fp16", "fp32", None)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kinds", KINDS, ids=str)
@pytest.mark.parametrize("shift", [0, 1])
def test_steps(L, kinds, bits, shift):
    params, grads, copies = tensors(ODD, *kinds, shift=shift)
    check_steps(AdamW(L, params, copies, bits), params, grads, copies, kinds)


@pytest.mark.parametrize("bits", [32, 8])
def test_scaled_gradients_and_other_rates(L, bits):
    params, grads, copies = tensors(ODD, "fp32", "fp16", "fp16", seed=3)
    scale = torch.tensor(2.0 ** -7 * 1.1, device="cuda")
    check_steps(AdamW(L, params, copies, bits), params, grads, copies, "scaled", scale, rate=0.5, beta1=0.0, beta2=0.9, eps=1e-3, decay=0.0)


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(L, bits):
    """More than one launch takes, of two kinds of types, in any order."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    params = [torch.randn(1 + 37 * i % 3000, generator=gen, device="cuda").to(torch.float32 if i % 3 else torch.bfloat16) for i in range(1203)]
    grads = [[torch.randn(p.shape, generator=gen, device="cuda").to(p.dtype) for p in params] for _ in range(2)]
    opt = AdamW(L, params, bits=bits)
    check_steps(opt, params, grads, None, "many")


def test_rounding_is_right_in_the_mean(L):
    """A v that a step would move by less than half a code's step does move, in the mean of its elements."""
    n = 1 << 20
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 1.0, device="cuda")
    opt = AdamW(L, [p], bits=8)
    steps = 100
    for _ in range(steps):
        opt.step([g], beta2=0.999)
    v = float(opt.moments()[1][0].double().mean())
    want = 1 - 0.999 ** steps
    # every step adds an error of at most one code's step (1/8 of a value of at most `want`) with mean 0: the mean over a million elements
    # of a hundred of them is off by less than want / 8 / 1000 * 10; 16 random bits put the mean off by 2^-17 of a step each time
    assert abs(v - want) < want * (6 * 10 / 8 / 1000 + steps / 8 * 2.0 ** -16)


def test_positive_second_moments_stay_positive(L):
    g = torch.zeros(512, device="cuda")
    g[0], g[1:256] = 1.0, 2.0 ** -19  # squares 2^-38 of the block's largest: below the smallest code's half
    opt = AdamW(L, [torch.zeros(512, device="cuda")], bits=8)
    opt.step([g])
    v = opt.moments()[1][0]
    assert bool((v[:256] > 0).all()) and not bool(v[256:].any())
    assert bool(torch.isfinite(opt.params[0]).all())


def test_a_bad_gradient_stays_in_its_block(L):
    params, grads, _ = tensors([(2000,)], "fp32", "fp32", steps=1)
    clean = params[0].clone()
    AdamW(L, [clean], bits=8).step(grads[0], seed=1)
    grads[0][0][300] = float("nan")
    opt = AdamW(L, params, bits=8)
    opt.step(grads[0], seed=1)
    m, v = opt.moments()
    for t in (m[0], v[0]):
        assert not bool(torch.isfinite(t[256:512]).any()) and bool(torch.isfinite(t[:256]).all()) and bool(torch.isfinite(t[512:]).all())
    keep = torch.arange(2000, device="cuda") != 300
    assert torch.equal(params[0][keep], clean[keep]) and bool(torch.isnan(params[0][300]))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-8, 1e-3, 1e-10, 0.0])
def test_ends_of_the_range(L, bits, eps):
    """Gradients whose squares are infinite, subnormal or 0 in fp32: an infinite second moment moves nothing, without eps the step's size is the rate."""
    size = [1e25, 1e10, 1.0, 1e-10, 1e-17] + ([] if eps == 0.0 else [1e-22, 0.0])
    g = torch.tensor(size, device="cuda").repeat_interleave(256)
    p = torch.ones_like(g)
    opt = AdamW(L, [p], bits=bits)
    opt.step([g], rate=0.25, decay=0.0, eps=eps)
    m, v = ref.moments_step(np.zeros(g.numel(), np.float32), np.zeros(g.numel(), np.float32), host(g), 0.9, 0.999)
    want, tol = ref.param_step(np.ones(g.numel(), np.float32), m, v, 0.25, 0.9, 0.999, np.float64(np.float32(eps)), 0.0, 1)
    # (a subnormal second moment keeps few digits, the same here and there; the smallest that 1e-17 leaves has 2^20 steps)
    assert (np.abs(host(p) - want) <= tol).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_scale_that_is_not_finite_leaves_all_as_it_was(L, bits):
    params, grads, copies = tensors(ODD, "fp32", "bf16", "bf16", steps=1)
    opt = AdamW(L, params, copies, bits)
    opt.step(grads[0])
    kept = [t.clone() for t in itertools.chain(params, copies, *opt.moments())]
    for bad in (float("inf"), float("nan"), -float("inf")):
        opt.step(grads[0], scale=torch.tensor([bad], device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip(kept, itertools.chain(params, copies, *opt.moments())))


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_count_on(L, bits):
    """A step in a graph with its number and rate on the device does what the same steps do outside."""
    shapes = [(300,), (40, 50)]
    params, grads, _ = tensors(shapes, "fp32", "fp32")
    others = [p.clone() for p in params]
    opt, plain = AdamW(L, params, bits=bits), AdamW(L, others, bits=bits)
    number, rate = torch.zeros(1, device="cuda", dtype=torch.int64), torch.zeros(1, device="cuda")
    held = [g.clone() for g in grads[0]]
    start = opt.state()
    keep = [p.clone() for p in params]
    number.fill_(1)
    opt.step(held, rate=rate, step=number, seed=5)  # (the workspace)
    for p, k in zip(params, keep):
        p.copy_(k)
    for some in start:
        for s in some:
            for t in s if bits == 8 else (s,):
                t.zero_()
    number.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        number += 1
        opt.step(held, rate=rate, step=number, seed=5)
    for k, some in enumerate(grads):
        for h, g in zip(held, some):
            h.copy_(g)
        rate.fill_(2.0 ** -(k + 5))
        graph.replay()
        plain.step(some, rate=2.0 ** -(k + 5), step=k + 1, seed=5 + k + 1)
    for a, b in zip(itertools.chain(params, *opt.moments()), itertools.chain(others, *plain.moments())):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [32, 8])
def test_state_goes_on_from_a_checkpoint(L, bits):
    params, grads, _ = tensors(ODD, "bf16", "bf16", steps=4)
    others = [p.clone() for p in params]
    whole = AdamW(L, params, bits=bits)
    for g in grads:
        whole.step(g)
    first = AdamW(L, others, bits=bits)
    for g in grads[:2]:
        first.step(g)
    second = AdamW(L, others, bits=bits)
    second.load(*first.state(), steps=first.steps)
    for g in grads[2:]:
        second.step(g)
    assert second.steps == 4
    for a, b in zip(itertools.chain(params, *whole.moments()), itertools.chain(others, *second.moments())):
        assert torch.equal(a, b)


def test_another_stream(L):
    params, grads, _ = tensors(ODD, "fp32", "fp32", steps=1)
    others = [p.clone() for p in params]
    opt, plain = AdamW(L, params, bits=8), AdamW(L, others, bits=8)
    plain.step(grads[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    opt.step(grads[0], stream=side)
    got = opt.moments(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(itertools.chain(params, *got), itertools.chain(others, *plain.moments())):
        assert torch.equal(a, b)


def test_last_elements_of_a_long_tensor(L):
    """Offsets beyond 2^32 bytes, and the random bits' block numbers."""
    n = (1 << 30) + 1000
    p = torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    g = torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    g[-700:] = torch.randn(700, device="cuda").bfloat16()
    opt = AdamW(L, [p], bits=8)
    opt.step([g], rate=0.5, decay=0.0, seed=4)
    m, v = ref.moments_step(np.zeros(700, np.float32), np.zeros(700, np.float32), host(g[-700:]), 0.9, 0.999)
    want, tol = ref.param_step(np.zeros(700, np.float32), m, v, 0.5, 0.9, 0.999, 1e-8, 0.0, 1)
    assert (np.abs(host(p[-700:]) - want) <= tol + 2.0 ** -8 * np.abs(want)).all()
    assert not bool(p[:-700].any())
    (codes, e), _ = opt.state()[0][0], None
    start = n - 700 - (n - 700) % 256
    r = ref._mix(np.arange(start >> 8, (n + 255) >> 8, dtype=np.uint64))
    r = ref._mix(r ^ np.uint64(4))
    j = np.arange(n - start, dtype=np.uint64)
    bits = ref._mix((r[(j >> np.uint64(8)).astype(np.int64)] + (j & np.uint64(255)) * np.uint64(0x6A09E667)) & np.uint64(ref.M32))
    whole = np.zeros(n - start, np.float32)
    whole[-700:] = m
    code, exponent = ref.encode(whole, True, bits)
    assert np.array_equal(codes[start:].cpu().numpy(), code) and np.array_equal(e[start >> 8:].cpu().numpy(), exponent)


def test_refusals(L):
    new = lambda *s, t=torch.float32: torch.zeros(*s, device="cuda", dtype=t)  # noqa: E731
    p, g = new(10), new(10)
    for bad in (lambda: AdamW(L, [p], bits=16), lambda: AdamW(L, [p, p]), lambda: AdamW(L, [p, p[2:]]), lambda: AdamW(L, [p.int()]), lambda: AdamW(L, [new(4, 4).t()[1:]]),
                lambda: AdamW(L, [p], copies=[g]), lambda: AdamW(L, [p.half()], copies=[p.half()]), lambda: AdamW(L, [p], copies=[]), lambda: AdamW(L, [p.cpu()]),
                lambda: AdamW(L, [p], copies=[new(9, t=torch.bfloat16)]), lambda: AdamW(L, [p]).step([]), lambda: AdamW(L, [p]).step([g[:5]]), lambda: AdamW(L, [p]).step([g.int()]),
                lambda: AdamW(L, [p]).step([new(20)[::2]]), lambda: AdamW(L, [p.half()]).step([g.bfloat16()]), lambda: AdamW(L, [p, new(3)]).step([g, new(3, t=torch.bfloat16)]),
                lambda: AdamW(L, [p]).step([g], step=0), lambda: AdamW(L, [p]).step([g], scale=new(2)), lambda: AdamW(L, [p]).step([g], scale=new(1, t=torch.bfloat16)),
                lambda: AdamW(L, [p]).step([g], step=torch.ones(1, device="cuda")), lambda: AdamW(L, [p]).step([g.cpu()]), lambda: AdamW(L, [p], bits=8).load([g], [g]),
                lambda: AdamW(L, [p]).load([], [])):
        with pytest.raises((TypeError, ValueError)):
            bad()
    for kw in ({"beta1": 1.0}, {"beta2": -0.1}, {"eps": -1.0}, {"decay": float("nan")}):
        with pytest.raises(SomError):
            AdamW(L, [p]).step([g], **kw)
    assert not bool(p.any())


def test_nothing_to_do(L):
    AdamW(L, []).step([])
    opt = AdamW(L, [torch.zeros(0, device="cuda")], bits=8)
    opt.step([torch.zeros(0, device="cuda")])
    assert opt.moments()[0][0].numel() == 0
