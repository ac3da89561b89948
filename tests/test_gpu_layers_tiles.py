"""GPU tests of the dense operators at sizes that reach every tile shape of their products, with more than one tile a block: what long
prompts, training steps and batches of single tokens run on; and of a few rows without tiles.  Bounds as in layers_reference.py; sums are kept short, the outputs large."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import layers_reference as ref  # noqa: E402
from test_gpu_layers import _expert_inputs, _linear_grad, _normal, _route, _wide  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture
def L():
    """A handle of the test's own: it has seen no other launches."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_24067_b200 import layers
    return layers.Layers()


def _linear_inputs(T, D, F, dtype, gated, wide):
    gen = torch.Generator().manual_seed(T + D + F)
    rows = 2 * F if gated else F
    return (_normal(gen, T, D, dtype=dtype, wide=wide), _normal(gen, rows, D, scale=D ** -0.5, dtype=dtype), _normal(gen, rows, dtype=dtype),
            _normal(gen, T, F, dtype=dtype, wide=wide))


@pytest.mark.parametrize("T,D,F", [(T, D, F) for T in (2, 3, 4, 6, 7, 8) for D, F in ((1032, 200), (72, 2504))] + [(3, 8200, 40), (5, 6552, 24)])
@pytest.mark.parametrize("dtype,act,gated,bias,residual,wide", [(BF16, "silu", True, True, True, 8), (FP16, "gelu", False, True, False, 0)])
def test_linear_few_rows(L, T, D, F, dtype, act, gated, bias, residual, wide):
    """Every number of rows that shares a read of the weights, long rows (few blocks an SM), and many outputs a warp."""
    x, w, b, r = _linear_inputs(T, D, F, dtype, gated, wide)
    b, r = b if bias else None, r if residual else None
    y = L.linear(x, w, b, r, act=act, gated=gated)
    h, eh, _, _ = ref.hidden(_wide(x), _wide(w), _wide(b), act, gated)
    if r is not None:
        h, eh = h + _wide(r), eh + 2.0 ** -22 * (h.abs() + _wide(r).abs())
    ref.close(y, h, ref.rounded(h, eh, dtype), "y")
    assert torch.equal(y, L.linear(x, w, b, r, act=act, gated=gated))
    assert all(L.rounds("forward", t) == 0 for t in ("128x128", "128x256", "256x256"))
    assert L.device_flags() == 0


@pytest.mark.parametrize("T,D,F,tiles", [(2, 1032, 8200, False), (2, 520, 20000, True), (4, 2048, 4096, False), (4, 2048, 8200, True),
                                         (8, 2048, 1024, False), (8, 2048, 4096, True), (8, 8192, 64, True)])
def test_linear_few_rows_or_tiles(L, T, D, F, tiles):
    """A few rows against many weights are the tiles' work (4 rows of 4096 against 8192 outputs: 26 us by rows, 23 by tiles; 8 rows 47 and
    22), against few weights the rows'."""
    x, w, _, _ = _linear_inputs(T, D, F, BF16, False, 0)
    y = L.linear(x, w)
    assert any(L.rounds("forward", t) for t in ("128x128", "128x256", "256x256")) == tiles
    z, ez = ref.product(_wide(x), torch.zeros_like(_wide(x)), _wide(w).t(), torch.zeros_like(_wide(w).t()))
    ref.close(y, z, ref.rounded(z, ez, BF16), "y")


@pytest.mark.parametrize("dtype,act,gated,bias,residual,wide", [
    (BF16, "gelu", False, True, True, 0), (FP16, "none", False, False, False, 8), (BF16, "silu", True, True, True, 16), (FP16, "relu", True, False, False, 0)])
def test_linear_pairs(L, dtype, act, gated, bias, residual, wide):
    T, D, F = 2605, 136, 1048 if gated else 2072
    x, w, b, r = _linear_inputs(T, D, F, dtype, gated, wide)
    b, r = b if bias else None, r if residual else None
    out = torch.zeros(T, F + wide, dtype=dtype, device="cuda")
    y = L.linear(x, w, b, r, act=act, gated=gated, out=out[:, :F])
    assert L.rounds("forward", "256x256") >= 2
    h, eh, _, _ = ref.hidden(_wide(x), _wide(w), _wide(b), act, gated)
    if r is not None:
        h, eh = h + _wide(r), eh + 2.0 ** -22 * (h.abs() + _wide(r).abs())
    ref.close(y, h, ref.rounded(h, eh, dtype), "y")
    assert not out[:, F:].any()
    assert torch.equal(y, L.linear(x, w, b, r, act=act, gated=gated))
    assert L.device_flags() == 0


# (dz in pairs; dx in pairs; dw in pairs)
@pytest.mark.parametrize("product,T,D,F", [("dz", 2605, 136, 2072), ("dx", 2605, 2072, 136), ("dw", 200, 2072, 2600)])
@pytest.mark.parametrize("dtype,act,gated,bias,wide", [
    (BF16, "gelu", False, True, 8), (FP16, "silu", False, False, 0), (BF16, "silu", True, True, 0), (FP16, "relu", True, True, 16)])
def test_linear_backward_pairs(L, product, T, D, F, dtype, act, gated, bias, wide):
    F = F // 16 * 8 if gated else F
    x, w, b, dy = _linear_inputs(T, D, F, dtype, gated, wide)
    b = b if bias else None
    got = L.linear_backward(x, w, dy, b, act=act, gated=gated)
    assert L.rounds(product, "256x256") >= 2
    want = _linear_grad(_wide(x), _wide(w), _wide(b), _wide(dy), act, gated, dtype)
    for n, v in got.items():
        ref.close(v, *want[n], n)
    again = L.linear_backward(x, w, dy, b, act=act, gated=gated)
    assert all(torch.equal(got[n], again[n]) for n in got)
    assert L.device_flags() == 0


# a few rows an expert; rows enough for pairs; few experts with few rows
EXPERTS = [("128x256", 96, 64, 6, 520, 264), ("256x256", 4000, 8, 2, 520, 520), ("128x128", 300, 40, 8, 512, 256)]


@pytest.mark.parametrize("tiles,T,E,k,D,I", EXPERTS)
@pytest.mark.parametrize("dtype,act,gated,bias,residual", [(BF16, "silu", True, False, True), (FP16, "gelu", False, True, False), (FP16, "silu", True, True, True)])
def test_experts_tiles(L, tiles, T, E, k, D, I, dtype, act, gated, bias, residual):
    gen = torch.Generator().manual_seed(T + E + D)
    s, r = _expert_inputs(T, E, k, D, I, dtype, gated, bias, residual, gen, FP32, pad=0.05)
    y = L.experts(s["x"], s["indices"], s["weights"], s["w1"], s["w2"], s["b1"], s["b2"], r, act=act, gated=gated)
    assert L.rounds("forward", tiles) >= 2 and all(L.rounds("forward", t) == 0 for t in {"128x128", "128x256", "256x256"} - {tiles})
    c = {n: _wide(v) for n, v in s.items()}
    want, bound = ref.experts(c["x"], s["indices"].cpu(), c["weights"], c["w1"], c["w2"], c["b1"], c["b2"], _wide(r), act, gated, dtype)
    ref.close(y, want, bound, "y")
    assert torch.equal(y, L.experts(s["x"], s["indices"], s["weights"], s["w1"], s["w2"], s["b1"], s["b2"], r, act=act, gated=gated))
    assert L.device_flags() == 0


@pytest.mark.parametrize("tiles,T,E,k,D,I", EXPERTS)
@pytest.mark.parametrize("dtype,act,gated,bias,wtype", [(BF16, "silu", True, True, FP32), (FP16, "gelu", False, True, FP16), (FP16, "silu", True, False, FP32)])
def test_experts_backward_tiles(L, tiles, T, E, k, D, I, dtype, act, gated, bias, wtype):
    gen = torch.Generator().manual_seed(T + E + D)
    s, _ = _expert_inputs(T, E, k, D, I, dtype, gated, bias, False, gen, wtype, pad=0.05)
    dy = _normal(gen, T, D, dtype=dtype, wide=8)
    got = L.experts_backward(s["x"], s["indices"], s["weights"], s["w1"], s["w2"], dy, s["b1"], s["b2"], act=act, gated=gated)
    assert L.rounds("dz of experts", tiles) >= 2 and L.rounds("dx", tiles) >= 2
    assert max(L.rounds("dw", t) for t in ("128x128", "256x256")) >= 2
    c = {n: _wide(v) for n, v in s.items()}
    want = ref.experts_backward(c["x"], s["indices"].cpu(), c["weights"], c["w1"], c["w2"], c["b1"], c["b2"], _wide(dy), act, gated, dtype)
    for n, v in got.items():
        ref.close(v, want[n][0], ref.rounded(*want[n], wtype) if n == "dweights" else want[n][1], n)
    again = L.experts_backward(s["x"], s["indices"], s["weights"], s["w1"], s["w2"], dy, s["b1"], s["b2"], act=act, gated=gated)
    assert all(torch.equal(got[n], again[n]) for n in got)
    assert L.device_flags() == 0


@pytest.mark.parametrize("T,E,k,opt,form", [
    (16400, 256, 8, dict(score="sigmoid", bias=True, groups=8, top_groups=4, group_best=2), "four lanes a token"),
    (16400, 128, 12, dict(score="sigmoid", renorm=False, bias=True, groups=4, top_groups=1, group_best=1), "four lanes a token"),
    (16400, 96, 5, dict(score="softmax", bias=True), "four lanes a token"),
    (16400, 64, 16, dict(score="softmax", bias=True, groups=2, top_groups=1, group_best=2, scale=2.5), "four lanes a token"),
    (16400, 512, 8, dict(score="softmax", renorm=False, bias=True, groups=8, top_groups=3, group_best=2), "four lanes a token"),
    (16400, 256, 8, dict(score="softmax", bias=True, groups=8, top_groups=4, group_best=2), "warp a token"),
    (8200, 512, 8, dict(score="sigmoid", bias=True, groups=16, top_groups=4, group_best=2), "four lanes a token"),
    (8200, 256, 8, dict(score="sigmoid", bias=True, groups=8, top_groups=4, group_best=2), "warp a token"),
    (8200, 200, 7, dict(score="softmax", renorm=False), "four lanes a token"),
    (8191, 200, 7, dict(score="softmax", renorm=False), "warp a token")])
@pytest.mark.parametrize("dtype,kind", [(FP32, "normal"), (BF16, "masked"), (FP32, "contested")])
def test_route_forms(L, T, E, k, opt, form, dtype, kind):
    """Both forms of the routing kernel on either side of the rule between them."""
    gen = torch.Generator().manual_seed(T + E)
    z = torch.randn(T, E, generator=gen) * 2
    bias = torch.randn(E, generator=gen) * 0.1 if opt.get("bias") else None
    if kind == "masked":
        z[torch.rand(z.shape, generator=gen) < 0.3] = -float("inf")
        z[::7] = -float("inf")
    if kind == "contested":
        z = z.round() / 2 + torch.randn(T, E, generator=gen) * 2.0 ** -20
        bias = None if bias is None else (bias * 32).round() / 32
    logits, opt = z.to(dtype).cuda(), {"renorm": True, **opt}
    got = L.route(logits, k, bias=None if bias is None else bias.cuda(), **{n: v for n, v in opt.items() if n != "bias"})
    assert L.rounds("route", form) >= 1 and sum(L.rounds("route", f) > 0 for f in ("warp a token", "four lanes a token")) == 1
    some = torch.arange(3, T, 83)
    _, (w, want, _, _) = _route(logits[some], k, opt, bias)
    assert torch.equal(got["indices"][some].cpu().long(), want)
    # exponentials, a sum of up to E of them and two divisions in fp32: (E + 16) half units
    assert ((got["weights"][some].double().cpu() - w).abs() <= (E + 16) * 2.0 ** -24 * w.abs() + 1e-37).all()
    at = got["indices"].long()
    assert torch.equal(got["counts"].long(), torch.bincount(at[at >= 0], minlength=E))
