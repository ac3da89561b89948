"""GPU tests of the dense operators (som_linear, som_route, som_experts and their gradients) against their definitions in
fp64; the bounds are derived in layers_reference.py."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import layers_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_24067_b200 import layers
    return layers.Layers()


def _normal(gen, *shape, scale=1.0, dtype=FP32, wide=0):
    """CPU values of dtype; wide > 0: rows of a matrix that is that much wider."""
    if wide:
        return (torch.randn(shape[0], shape[1] + wide, generator=gen) * scale).to(dtype).cuda()[:, :shape[1]]
    return (torch.randn(*shape, generator=gen) * scale).to(dtype).cuda()


def _wide(t):
    return None if t is None else t.double().cpu()


SIZES = [(1, 8, 8), (1, 64, 128), (2, 72, 40), (5, 2048, 264), (16, 136, 520), (17, 200, 256), (64, 64, 64), (127, 136, 264),
         (128, 256, 256), (129, 264, 136), (300, 520, 1000),
         (40, 2048, 264), (200, 3000, 72), (3000, 72, 72), (9, 1000, 4096)]  # (sums split over blocks)


@pytest.mark.parametrize("T,D,F", SIZES)
@pytest.mark.parametrize("dtype,act,gated,bias,residual,wide", [
    (BF16, "none", False, False, False, 0), (FP16, "relu", False, True, True, 8), (BF16, "gelu", False, True, False, 0),
    (FP16, "silu", True, True, True, 24), (BF16, "silu", True, False, False, 0), (FP16, "gelu", True, False, True, 8),
    (BF16, "none", True, True, False, 16)])
def test_linear(L, T, D, F, dtype, act, gated, bias, residual, wide):
    gen = torch.Generator().manual_seed(T * 7 + D + F)
    rows = 2 * F if gated else F
    x = _normal(gen, T, D, dtype=dtype, wide=wide)
    w = _normal(gen, rows, D, scale=D ** -0.5, dtype=dtype)
    b = _normal(gen, rows, dtype=dtype) if bias else None
    r = _normal(gen, T, F, dtype=dtype, wide=wide) if residual else None
    out = torch.zeros(T, F + wide, dtype=dtype, device="cuda")
    y = L.linear(x, w, b, r, act=act, gated=gated, out=out[:, :F])
    h, eh, _, _ = ref.hidden(_wide(x), _wide(w), _wide(b), act, gated)
    if r is not None:
        h, eh = h + _wide(r), eh + 2.0 ** -22 * (h.abs() + _wide(r).abs())
    ref.close(y, h, ref.rounded(h, eh, dtype), "y")
    assert not out[:, F:].any()  # what lies between the rows is not written
    assert torch.equal(y, L.linear(x, w, b, r, act=act, gated=gated))
    assert L.device_flags() == 0


def _linear_grad(x, w, b, dy, act, gated, dtype):
    h, eh, z, ez = ref.hidden(x, w, b, act, gated)
    dz, edz = ref.hidden_grad(z, ez, dy, torch.zeros_like(dy), act, gated)
    if act == "none" and not gated:
        zz = torch.zeros_like(dz)
    else:
        zz = ref.rounded(dz, edz + 2.0 ** -21 * dz.abs(), dtype)
    dx, edx = ref.product(dz, zz, w, torch.zeros_like(w))
    dw, edw = ref.product(dz.t(), zz.t(), x, torch.zeros_like(x))
    db, edb = dz.sum(0), zz.sum(0) + x.shape[0] * 2.0 ** -23 * dz.abs().sum(0)
    return {"dx": (dx, ref.rounded(dx, edx, dtype)), "dweight": (dw, ref.rounded(dw, edw, dtype)), "dbias": (db, ref.rounded(db, edb, dtype))}


@pytest.mark.parametrize("T,D,F", SIZES)
@pytest.mark.parametrize("dtype,act,gated,bias,wide", [
    (BF16, "none", False, True, 8), (FP16, "relu", False, True, 0), (BF16, "gelu", False, True, 0), (FP16, "silu", False, False, 16),
    (BF16, "silu", True, True, 0), (FP16, "gelu", True, True, 8), (BF16, "relu", True, False, 0), (FP16, "none", True, True, 0)])
def test_linear_backward(L, T, D, F, dtype, act, gated, bias, wide):
    gen = torch.Generator().manual_seed(T * 5 + D + F)
    rows = 2 * F if gated else F
    x = _normal(gen, T, D, dtype=dtype, wide=wide)
    w = _normal(gen, rows, D, scale=D ** -0.5, dtype=dtype)
    b = _normal(gen, rows, dtype=dtype) if bias else None
    dy = _normal(gen, T, F, dtype=dtype, wide=wide)
    got = L.linear_backward(x, w, dy, b, act=act, gated=gated)
    want = _linear_grad(_wide(x), _wide(w), _wide(b), _wide(dy), act, gated, dtype)
    for n, v in got.items():
        ref.close(v, *want[n], n)
    again = L.linear_backward(x, w, dy, b, act=act, gated=gated)
    assert all(torch.equal(got[n], again[n]) for n in got)
    assert L.device_flags() == 0


@pytest.mark.parametrize("act,gated", [("gelu", False), ("silu", True), ("none", True)])
def test_linear_backward_against_differences(L, act, gated):
    """<gradient, direction> against the central difference of the fp64 definition along that direction.  The gradients are
    16-bit numbers from operands rounded to 16 bits: their inner product with a fixed direction is off by at most
    2 * 2^-11 * sum of magnitudes; the difference's own error (step 1e-5) is far below."""
    gen = torch.Generator().manual_seed(5)
    T, D, F = 37, 72, 48
    rows = 2 * F if gated else F
    x, w = _normal(gen, T, D, dtype=FP16), _normal(gen, rows, D, scale=D ** -0.5, dtype=FP16)
    b, dy = _normal(gen, rows, dtype=FP16), _normal(gen, T, F, dtype=FP16)
    got = L.linear_backward(x, w, dy, b, act=act, gated=gated)
    at = {"dx": _wide(x), "dweight": _wide(w), "dbias": _wide(b)}

    def loss(v):
        return (ref.hidden(v["dx"], v["dweight"], v["dbias"], act, gated)[0] * _wide(dy)).sum()

    mags = _linear_grad(_wide(x), _wide(w), _wide(b), _wide(dy), act, gated, FP16)
    for n in at:
        d = torch.randn(at[n].shape, generator=gen, dtype=torch.float64)
        step = 1e-5
        diff = (loss({**at, n: at[n] + step * d}) - loss({**at, n: at[n] - step * d})) / (2 * step)
        bound = (mags[n][1] * d.abs()).sum() + 1e-6 * diff.abs()
        assert abs(float((got[n].double().cpu() * d).sum() - diff)) <= float(bound), n


def test_linear_keeps_rows_apart(L):
    """A token with NaN, or with infinities, changes no other token's row; weights' NaN stay in their own column."""
    gen = torch.Generator().manual_seed(9)
    for T in (3, 200):
        x, w = _normal(gen, T, 72, dtype=BF16), _normal(gen, 136, 72, dtype=BF16)
        clean = L.linear(x, w, act="silu")
        x2, w2 = x.clone(), w.clone()
        x2[1] = math.nan
        x2[2, 3] = math.inf
        w2[7] = math.nan
        y = L.linear(x2, w2, act="silu")
        rows = [i for i in range(T) if i not in (1, 2)]
        cols = [i for i in range(136) if i != 7]
        assert torch.equal(y[rows][:, cols], clean[rows][:, cols])
        assert y[1].isnan().all() and y[:, 7].isnan().all()


def test_linear_on_another_stream(L):
    gen = torch.Generator().manual_seed(3)
    x, w = _normal(gen, 100, 256, dtype=BF16), _normal(gen, 512, 256, dtype=BF16)
    want = L.linear(x, w, act="gelu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = L.linear(x, w, act="gelu", stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    with torch.cuda.stream(side):
        got = L.linear(x, w, act="gelu")
    side.synchronize()
    assert torch.equal(got, want)


# ---- routing ---------------------------------------------------------------------------------------------------

ROUTES = [dict(score="softmax", renorm=True), dict(score="softmax", renorm=False, scale=2.5), dict(score="sigmoid", renorm=True),
          dict(score="sigmoid", renorm=False), dict(score="softmax", renorm=True, bias=True), dict(score="sigmoid", renorm=True, bias=True, scale=1.5),
          dict(score="softmax", renorm=False, groups=4, top_groups=2), dict(score="sigmoid", renorm=True, bias=True, groups=4, top_groups=1, group_best=2),
          dict(score="sigmoid", renorm=False, groups=2, top_groups=1, group_best=2)]


def _route(logits, k, opt, bias):
    o = {"groups": 1, "top_groups": 1, "group_best": 1, "scale": 1.0, **{n: v for n, v in opt.items() if n != "bias"}}
    return o, ref.route(logits.float().cpu(), k, o["score"], None if bias is None else bias.cpu(), o["groups"], o["top_groups"], o["group_best"], o["renorm"], o["scale"])


@pytest.mark.parametrize("T,E,k", [(1, 4, 1), (1, 64, 8), (3, 8, 8), (33, 36, 4), (70, 100, 6), (9, 256, 12), (5, 516, 3), (4, 1024, 32)])
@pytest.mark.parametrize("opt", ROUTES)
@pytest.mark.parametrize("dtype,kind", [(FP32, "normal"), (BF16, "normal"), (FP16, "masked"), (FP32, "ties"), (FP32, "wild")])
def test_route(L, T, E, k, opt, dtype, kind):
    gen = torch.Generator().manual_seed(T + E + k)
    z = torch.randn(T, E + 3, generator=gen) * 2
    if kind == "ties":
        z = z.round().clamp(-1, 1) * 0.0 if T == 1 else z.round().clamp(-1, 1)  # many equal logits, of both signs of zero
    if kind == "masked":
        z[torch.rand(z.shape, generator=gen) < 0.3] = -math.inf
        z[::3] = -math.inf  # rows whose mask leaves nothing
    if kind == "wild":
        z[:, 1] = math.inf
        z[:, 2] = math.nan
        z[::2, 3] = -1e30
        z[1::2, 0] = torch.finfo(FP32).min  # fp32's lowest value is a number, not a mask
    logits = z.to(dtype).cuda()[:, 1:E + 1] if kind != "wild" else z.to(dtype).cuda()[:, :E]  # odd offsets, rows apart
    bias = (torch.randn(E, generator=gen) * 0.3).cuda() if opt.get("bias") else None
    o, (w, at, counts, _) = _route(logits, k, opt, bias)
    got = L.route(logits, k, bias=bias, **o)
    assert torch.equal(got["indices"].cpu().long(), at)
    assert torch.equal(got["counts"].cpu().long(), counts)
    # exponentials, a sum of up to E of them and two divisions in fp32: (E + 16) half units
    assert ((got["weights"].double().cpu() - w).abs() <= (E + 16) * 2.0 ** -24 * w.abs() + 1e-37).all()
    again = L.route(logits, k, bias=bias, **o)
    assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("E,k,opt", [
    (64, 8, dict(score="softmax", renorm=True)), (100, 6, dict(score="softmax", renorm=False)), (8, 8, dict(score="sigmoid", renorm=True)),
    (256, 8, dict(score="sigmoid", renorm=True, bias=True, groups=8, top_groups=4, group_best=2)), (300, 16, dict(score="softmax", renorm=True, bias=True)),
    (128, 12, dict(score="softmax", renorm=True, groups=4, top_groups=2)), (1024, 9, dict(score="sigmoid", renorm=False, bias=True, groups=32, top_groups=3, group_best=1)),
    (36, 2, dict(score="sigmoid", renorm=True, groups=2, top_groups=1)), (64, 20, dict(score="softmax", renorm=True)), (1, 1, dict(score="softmax", renorm=True))])
@pytest.mark.parametrize("dtype,kind", [(FP32, "normal"), (BF16, "normal"), (FP16, "masked"), (FP32, "ties")])
def test_route_many_tokens(L, E, k, opt, dtype, kind):
    """Many tokens take another form of the kernel: the choice is that of the same tokens a few at a time, and of the definition."""
    T = 8201
    gen = torch.Generator().manual_seed(E + k)
    z = torch.randn(T, E, generator=gen) * 2
    if kind == "ties":
        z = (z * 2).round() / 2
    if kind == "masked":
        z[torch.rand(z.shape, generator=gen) < 0.3] = -math.inf
        z[::7] = -math.inf
    logits = z.to(dtype).cuda()
    bias = (torch.randn(E, generator=gen) * 0.1).cuda() if opt.get("bias") else None
    got = L.route(logits, k, bias=bias, **{n: v for n, v in opt.items() if n != "bias"})
    at = torch.cat([L.route(logits[i:i + 600], k, bias=bias, **{n: v for n, v in opt.items() if n != "bias"})["indices"] for i in range(0, T, 600)])
    assert torch.equal(got["indices"], at)
    assert torch.equal(got["counts"].long(), torch.bincount(at[at >= 0].long(), minlength=E))
    some = torch.arange(3, T, 61)
    _, (w, want, _, _) = _route(logits[some], k, opt, bias)
    assert torch.equal(got["indices"][some].cpu().long(), want)
    assert ((got["weights"][some].double().cpu() - w).abs() <= (E + 16) * 2.0 ** -24 * w.abs() + 1e-37).all()
    again = L.route(logits, k, bias=bias, **{n: v for n, v in opt.items() if n != "bias"})
    assert all(torch.equal(got[n], again[n]) for n in got)


def test_route_order_of_near_scores(L):
    """Scores that differ by less than one fp32 exponential's error are ordered as their fp32 roundings from 64 bits are."""
    gen = torch.Generator().manual_seed(0)
    base = torch.rand(400, 1, generator=gen) * 4 - 2
    z = (base + torch.arange(16) * 2.0 ** -22).float()
    z = z[:, torch.randperm(16, generator=gen)].contiguous()
    for score in ("sigmoid", "softmax"):
        bias = torch.zeros(16)
        _, at, _, _ = ref.route(z, 5, score, bias, 1, 1, 1, True, 1.0)
        assert torch.equal(L.route(z.cuda(), 5, score=score, bias=bias.cuda())["indices"].cpu().long(), at)


@pytest.mark.parametrize("T", [350, 8200])
@pytest.mark.parametrize("groups,top_groups,group_best", [(1, 1, 1), (4, 2, 2), (4, 3, 1)])
@pytest.mark.parametrize("score,spread", [("sigmoid", 2.0 ** -22), ("sigmoid", 2.0 ** -18), ("softmax", 2.0 ** -20)])
def test_route_contested(L, T, score, spread, groups, top_groups, group_best):
    """The same in both forms of the kernel: values from a coarse grid plus noise far below it, so that choices, boundaries and groups are
    contested in every token, some by two experts and some by many."""
    gen = torch.Generator().manual_seed(7)
    T, E, k = T, 128, 8
    z = (torch.randn(T, E, generator=gen) * 4).round() / 4 + torch.randn(T, E, generator=gen) * spread
    bias = (torch.randn(E, generator=gen) * 4).round() / 64
    got = L.route(z.cuda(), k, score=score, bias=bias.cuda(), groups=groups, top_groups=top_groups, group_best=group_best)
    some = torch.arange(0, T, 1 + T // 350)
    _, at, _, _ = ref.route(z[some], k, score, bias, groups, top_groups, group_best, True, 1.0)
    assert torch.equal(got["indices"][some].cpu().long(), at)


@pytest.mark.parametrize("T,E,k", [(1, 4, 2), (33, 36, 4), (70, 100, 6), (9, 256, 12), (4, 1024, 32), (2, 1, 1)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_route_backward(L, T, E, k, score, renorm, dtype):
    gen = torch.Generator().manual_seed(T + E)
    z = torch.randn(T, E + 1, generator=gen)
    if E > 8:
        z[torch.rand(z.shape, generator=gen) < 0.2] = -math.inf
        z[::4] = -math.inf
    logits = z.to(dtype).cuda()[:, :E]
    at = L.route(logits, k, score=score, renorm=renorm, scale=1.5)["indices"]
    dw = torch.randn(T, k, generator=gen)
    got = L.route_backward(logits, at, dw.cuda(), score=score, renorm=renorm, scale=1.5).double().cpu()
    x = logits.double().cpu()
    dead = x == -math.inf
    x = x.masked_fill(dead, -1e5).requires_grad_()
    s = torch.sigmoid(x) if score == "sigmoid" else torch.softmax(x, 1)
    idx = at.cpu().long()
    w = s.gather(1, idx.clamp_min(0)) * (idx >= 0)
    if renorm:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    (1.5 * w * dw.double()).sum().backward()
    want = x.grad.masked_fill(dead, 0)
    # every gradient is a score times a difference of (weighted means of) dweights, all in fp32
    size = 1.5 * dw.double().abs().max(1, keepdim=True).values * (s.detach() if not renorm else 1.0).clamp_max(1.0) if not renorm else 1.5 * dw.double().abs().max(1, keepdim=True).values
    bound = (E + 3 * k + 32) * 2.0 ** -23 * size + (0 if dtype == FP32 else 2.0 ** -8 * want.abs())
    assert ((got - want).abs() <= bound).all()
    assert (got[dead] == 0).all()


def test_route_backward_against_differences(L):
    gen = torch.Generator().manual_seed(1)
    z = torch.randn(20, 24, generator=gen, dtype=torch.float64).float()
    d = torch.randn(20, 24, generator=gen, dtype=torch.float64)
    dw = torch.randn(20, 4, generator=gen)
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            at = L.route(z.cuda(), 4, score=score, renorm=renorm)["indices"]
            g = L.route_backward(z.cuda(), at, dw.cuda(), score=score, renorm=renorm).double().cpu()

            def loss(x):
                s = torch.sigmoid(x) if score == "sigmoid" else torch.softmax(x, 1)
                w = s.gather(1, at.cpu().long())
                return ((w / w.sum(1, keepdim=True) if renorm else w) * dw.double()).sum()

            step = 1e-5
            diff = (loss(z.double() + step * d) - loss(z.double() - step * d)) / (2 * step)
            # 480 fp32 numbers of magnitude at most 6, each off by at most 64 half units, against d of magnitude at most 4
            assert abs(float((g * d).sum() - diff)) < 480 * 6 * 4 * 64 * 2.0 ** -24


def test_route_backward_bad_and_repeated_indices(L):
    z = torch.randn(6, 10, generator=torch.Generator().manual_seed(2)).cuda()
    at = torch.tensor([[0, 1], [1, -1], [3, 10], [-7, 2], [4, 4], [-1, -1]], dtype=torch.int32).cuda()
    dw = torch.ones(6, 2, device="cuda")
    g = L.route_backward(z, at, dw, score="sigmoid", renorm=False)
    assert L.device_flags() == 1 and L.device_flags() == 0
    s = torch.sigmoid(z.double())
    want = torch.zeros(6, 10, dtype=torch.float64, device="cuda")
    for t, e, n in ((0, 0, 1), (0, 1, 1), (1, 1, 1), (2, 3, 1), (3, 2, 1), (4, 4, 2)):
        want[t, e] = n * s[t, e] * (1 - s[t, e])
    assert torch.allclose(g.double(), want, rtol=1e-6, atol=0)


# ---- experts ---------------------------------------------------------------------------------------------------

CASES = [  # T, E, k, D, I
    (1, 4, 2, 64, 64), (1, 64, 8, 256, 136), (2, 5, 5, 72, 40), (7, 3, 1, 520, 264), (40, 16, 4, 264, 136), (130, 1, 1, 136, 200),
    (200, 5, 2, 264, 72), (300, 40, 8, 64, 128), (513, 6, 2, 256, 256),
    (1100, 7, 2, 264, 136)]


def _expert_inputs(T, E, k, D, I, dtype, gated, bias, residual, gen, wtype, pad=0.1):
    rows = 2 * I if gated else I
    z = torch.rand(T, E, generator=gen)
    z[:, 0] += 0.3  # one expert has most tokens
    at = z.topk(k, dim=1).indices
    none = torch.rand(T, k, generator=gen) < pad
    at[none] = -1
    if T > 6:
        at[3] = -1  # a token without an expert
    s = {"x": _normal(gen, T, D, dtype=dtype, wide=8), "indices": at.int().cuda(), "weights": torch.rand(T, k, generator=gen).to(wtype).cuda(),
         "w1": _normal(gen, E, rows, D, scale=D ** -0.5, dtype=dtype), "w2": _normal(gen, E, D, I, scale=I ** -0.5, dtype=dtype),
         "b1": _normal(gen, E, rows, scale=0.3, dtype=dtype) if bias else None, "b2": _normal(gen, E, D, scale=0.3, dtype=dtype) if bias else None}
    r = _normal(gen, T, D, dtype=dtype, wide=16) if residual else None
    return s, r


@pytest.mark.parametrize("T,E,k,D,I", CASES)
@pytest.mark.parametrize("dtype,act,gated,bias,residual", [
    (BF16, "silu", True, False, False), (FP16, "gelu", False, True, True), (BF16, "relu", True, True, True), (FP16, "silu", True, True, False)])
def test_experts(L, T, E, k, D, I, dtype, act, gated, bias, residual):
    gen = torch.Generator().manual_seed(T + E + D)
    s, r = _expert_inputs(T, E, k, D, I, dtype, gated, bias, residual, gen, FP32 if T % 2 else dtype)
    y = L.experts(s["x"], s["indices"], s["weights"], s["w1"], s["w2"], s["b1"], s["b2"], r, act=act, gated=gated)
    c = {n: _wide(v) for n, v in s.items()}
    want, bound = ref.experts(c["x"], s["indices"].cpu(), c["weights"], c["w1"], c["w2"], c["b1"], c["b2"], _wide(r), act, gated, dtype)
    ref.close(y, want, bound, "y")
    empty = (s["indices"] < 0).all(1)
    assert torch.equal(y[empty], torch.zeros_like(y[empty]) if r is None else r[empty])
    again = L.experts(s["x"], s["indices"], s["weights"], s["w1"], s["w2"], s["b1"], s["b2"], r, act=act, gated=gated)
    assert torch.equal(y, again)
    assert L.device_flags() == 0


@pytest.mark.parametrize("T,E,k,D,I", CASES)
@pytest.mark.parametrize("dtype,act,gated,bias,wtype", [
    (BF16, "silu", True, False, BF16), (FP16, "gelu", False, True, FP16), (BF16, "relu", True, True, FP32), (FP16, "silu", False, False, FP32),
    (FP16, "gelu", True, True, FP16)])
def test_experts_backward(L, T, E, k, D, I, dtype, act, gated, bias, wtype):
    gen = torch.Generator().manual_seed(T + E + D)
    s, _ = _expert_inputs(T, E, k, D, I, dtype, gated, bias, False, gen, wtype)
    dy = _normal(gen, T, D, dtype=dtype, wide=24)
    got = L.experts_backward(s["x"], s["indices"], s["weights"], s["w1"], s["w2"], dy, s["b1"], s["b2"], act=act, gated=gated)
    c = {n: _wide(v) for n, v in s.items()}
    want = ref.experts_backward(c["x"], s["indices"].cpu(), c["weights"], c["w1"], c["w2"], c["b1"], c["b2"], _wide(dy), act, gated, dtype)
    for n, v in got.items():
        ref.close(v, want[n][0], ref.rounded(*want[n], wtype) if n == "dweights" else want[n][1], n)
    unused = [e for e in range(E) if not (s["indices"] == e).any()]
    assert not got["dw1"][unused].any() and not got["dw2"][unused].any()
    again = L.experts_backward(s["x"], s["indices"], s["weights"], s["w1"], s["w2"], dy, s["b1"], s["b2"], act=act, gated=gated)
    assert all(torch.equal(got[n], again[n]) for n in got)
    assert L.device_flags() == 0


def test_experts_backward_against_differences(L):
    """As test_linear_backward_against_differences, over every input of the layer."""
    gen = torch.Generator().manual_seed(8)
    s, _ = _expert_inputs(30, 4, 2, 64, 40, FP16, True, True, False, gen, FP32)
    dy = _normal(gen, 30, 64, dtype=FP16)
    got = L.experts_backward(s["x"], s["indices"], s["weights"], s["w1"], s["w2"], dy, s["b1"], s["b2"], act="silu", gated=True)
    c = {n: _wide(v) for n, v in s.items()}
    at = s["indices"].cpu()
    want = ref.experts_backward(c["x"], at, c["weights"], c["w1"], c["w2"], c["b1"], c["b2"], _wide(dy), "silu", True, FP16)

    def loss(v):
        return (ref.experts(v["x"], at, v["weights"], v["w1"], v["w2"], v["b1"], v["b2"], None, "silu", True, FP16)[0] * _wide(dy)).sum()

    for n in ("x", "weights", "w1", "w2", "b1", "b2"):
        d = torch.randn(c[n].shape, generator=gen, dtype=torch.float64)
        if n == "weights":
            d = d * (at >= 0)
        step = 1e-5
        diff = (loss({**c, n: c[n] + step * d}) - loss({**c, n: c[n] - step * d})) / (2 * step)
        bound = ((want["d" + n][1] + 2.0 ** -23 * want["d" + n][0].abs()) * d.abs()).sum() + 1e-6 * diff.abs()
        assert abs(float((got["d" + n].double().cpu() * d).sum() - diff)) <= float(bound), n


def test_experts_bad_index_and_nan(L):
    """An index out of range counts as none and is recorded; NaN in a token or in an expert nobody chose stays there."""
    gen = torch.Generator().manual_seed(4)
    s, _ = _expert_inputs(150, 5, 2, 72, 64, BF16, True, True, False, gen, FP32, pad=0.0)
    at = s["indices"].clone()
    at[at == 4] = -1  # nobody chooses expert 4
    args = lambda i, x, w1: (x, i, s["weights"], w1, s["w2"], s["b1"], s["b2"])  # noqa: E731
    clean = L.experts(*args(at, s["x"], s["w1"]))
    grads = L.experts_backward(s["x"], at, s["weights"], s["w1"], s["w2"], s["x"], s["b1"], s["b2"])
    bad = at.clone()
    bad[at == -1] = 5
    bad[0][at[0] == -1] = -2
    assert torch.equal(L.experts(*args(bad, s["x"], s["w1"])), clean)
    assert L.device_flags() == 1
    x, w1 = s["x"].clone(), s["w1"].clone()
    x[11] = math.nan
    w1[4] = math.nan
    y = L.experts(*args(at, x, w1))
    keep = [t for t in range(150) if t != 11]
    assert torch.equal(y[keep], clean[keep]) and (y[11].isnan().all() or (at[11] < 0).all())
    g = L.experts_backward(x, at, s["weights"], w1, s["w2"], s["x"], s["b1"], s["b2"])
    assert torch.equal(g["dx"][keep], grads["dx"][keep])
    for e in range(5):
        if e not in at[11].tolist():
            assert torch.equal(g["dw1"][e], grads["dw1"][e]) and torch.equal(g["dw2"][e], grads["dw2"][e])


def test_no_tokens(L):
    x = torch.zeros(0, 64, dtype=BF16, device="cuda")
    w1, w2 = torch.ones(3, 32, 64, dtype=BF16, device="cuda"), torch.ones(3, 64, 16, dtype=BF16, device="cuda")
    none = torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    assert L.linear(x, w1[0]).shape == (0, 32)
    g = L.linear_backward(x, w1[0], torch.zeros(0, 32, dtype=BF16, device="cuda"), w1[0, :, 0].contiguous())
    assert not g["dweight"].any() and not g["dbias"].any()
    r = L.route(torch.zeros(0, 8, device="cuda"), 2)
    assert r["indices"].shape == (0, 2) and not r["counts"].any()
    assert L.route_backward(torch.zeros(0, 8, device="cuda"), none, torch.zeros(0, 2, device="cuda")).shape == (0, 8)
    assert L.experts(x, none, torch.zeros(0, 2, device="cuda"), w1, w2).shape == (0, 64)
    g = L.experts_backward(x, none, torch.zeros(0, 2, device="cuda"), w1, w2, x, w1[:, :, 0].contiguous(), w2[:, :, 0].contiguous())
    assert not any(g[n].any() for n in ("dw1", "dw2", "db1", "db2"))


def test_refusals(L):
    from paper_2608_24067_b200.som import SomError
    ok = torch.zeros(4, 64, dtype=BF16, device="cuda")
    w = torch.zeros(32, 64, dtype=BF16, device="cuda")

    def raises(kind, f, *a, status=None, **kw):
        with pytest.raises(kind) as e:
            f(*a, **kw)
        if status is not None:
            assert e.value.status == status

    raises(TypeError, L.linear, ok.float(), w)
    raises((TypeError, ValueError), L.linear, ok.cpu(), w)
    raises(TypeError, L.linear, ok, w.half())
    raises(ValueError, L.linear, ok, w[:, :32].contiguous())
    raises(TypeError, L.linear, ok, w[:, ::2])
    raises(TypeError, L.linear, ok.t(), w)
    raises(ValueError, L.linear, ok, w, act="tanh")
    raises(ValueError, L.linear, ok, w[:31], gated=True)
    raises(ValueError, L.linear, ok, w, residual=ok)
    raises(SomError, L.linear, torch.zeros(4, 60, dtype=BF16, device="cuda"), torch.zeros(32, 60, dtype=BF16, device="cuda"), status=3)
    raises(SomError, L.linear, ok, w[:31], status=3)
    raises(SomError, L.linear, torch.zeros(4, 72, dtype=BF16, device="cuda")[:, 1:65], w, status=3)  # rows off the 16-byte grid
    raises(SomError, L.linear, torch.zeros(4, 67, dtype=BF16, device="cuda")[:, :64], w, status=3)
    z = torch.zeros(4, 8, device="cuda")
    raises(SomError, L.route, z, 9, status=1)
    raises(SomError, L.route, z, 0, status=1)
    raises(SomError, L.route, z, 2, groups=3, status=1)
    raises(SomError, L.route, z, 2, groups=2, top_groups=3, status=1)
    raises(SomError, L.route, z, 2, groups=2, group_best=3, status=1)
    raises(SomError, L.route, torch.zeros(2, 1025, device="cuda"), 2, status=3)
    raises(SomError, L.route, torch.zeros(2, 64, device="cuda"), 33, status=3)
    raises(ValueError, L.route, z, 2, score="hardmax")
    raises(ValueError, L.route, z.double(), 2)
    raises(TypeError, L.route, z, 2, bias=z[0].half())
    at, wt = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    w1, w2 = torch.zeros(3, 32, 64, dtype=BF16, device="cuda"), torch.zeros(3, 64, 16, dtype=BF16, device="cuda")
    raises(TypeError, L.experts, ok, at.long(), wt, w1, w2)
    raises(TypeError, L.experts, ok, at, wt.half(), w1, w2)
    raises(ValueError, L.experts, ok, at, wt[:, :1].contiguous(), w1, w2)
    raises(ValueError, L.experts, ok, at, wt, w1, w2[:, :, :8].contiguous())
    raises(ValueError, L.experts, ok, at, wt, w1, w2, b1=w1[0])
    raises(SomError, L.experts, ok, at, wt, torch.zeros(3, 24, 64, dtype=BF16, device="cuda"), torch.zeros(3, 64, 12, dtype=BF16, device="cuda"), status=3)
    raises(ValueError, L.experts_backward, ok, at, wt, w1, w2, ok[:2])


def test_captured(L):
    """Routing, experts and their gradient replayed from a graph, with other inputs in the same tensors."""
    gen = torch.Generator().manual_seed(5)
    T, E, k, D, I = 70, 9, 3, 136, 72
    s, _ = _expert_inputs(T, E, k, D, I, BF16, True, True, False, gen, FP32)
    logits, dy = torch.randn(T, E, generator=gen).cuda(), _normal(gen, T, D, dtype=BF16)

    def step():
        r = L.route(logits, k, score="sigmoid", renorm=True)
        y = L.experts(s["x"], r["indices"], r["weights"], s["w1"], s["w2"], s["b1"], s["b2"], act="silu", gated=True)
        g = L.experts_backward(s["x"], r["indices"], r["weights"], s["w1"], s["w2"], dy, s["b1"], s["b2"], act="silu", gated=True)
        z = L.linear(y, s["w1"][0], act="gelu")
        return [r["indices"], r["weights"], y, z] + [g[n] for n in sorted(g)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for turn in range(2):
        logits.copy_(torch.randn(T, E, generator=gen))
        dy.copy_(torch.randn(T, D, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(kept, step()):
            assert torch.equal(a, b)
