"""GPU tests of how the dense operators are used: other streams, biases that switch experts off or are large,
values near the ends of fp16."""
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


def _choice(z, bias, k, score, groups, top_groups, group_best):
    """The k experts of the largest keys, best first, and their scores, from fp64; a key of -inf or NaN is never chosen and has no
    part in its group's key."""
    E = z.shape[1]
    z = z.double()
    s = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(z, 1)
    key = (s.float() + bias).masked_fill(z == -math.inf, -math.inf)
    key = key.masked_fill(key.isnan(), -math.inf)
    indices = torch.full((len(z), k), -1)
    for t in range(len(z)):
        row = key[t].tolist()
        rank = []
        for g in range(groups):
            best = sorted((v for v in row[g * (E // groups):(g + 1) * (E // groups)] if v > -math.inf), reverse=True)[:group_best]
            rank.append((-float(torch.tensor(best).sum()) if best else math.inf, g))
        kept = {g for v, g in sorted(rank)[:top_groups] if v < math.inf}
        of = sorted((i for i in range(E) if row[i] > -math.inf and i // (E // groups) in kept), key=lambda i: (-row[i], i))[:k]
        indices[t, :len(of)] = torch.tensor(of, dtype=torch.int64)
    return indices, s.gather(1, indices.clamp_min(0)) * (indices >= 0)


SWITCHES = [(64, 6, 1, 1, 1), (128, 8, 4, 2, 2), (128, 8, 4, 2, 1), (256, 12, 8, 3, 2), (100, 9, 1, 1, 1)]


@pytest.mark.parametrize("T", [1, 97, 12301])
@pytest.mark.parametrize("E,k,groups,top_groups,group_best", SWITCHES)
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("off", [-math.inf, math.nan])
def test_route_bias_switches_off(L, T, E, k, groups, top_groups, group_best, score, dtype, off):
    """An expert whose bias is -inf is never chosen, also where fewer than k others are left, and has no part in its group's key; NaN the
    same.  An infinite bias of the other sign is chosen first."""
    gen = torch.Generator().manual_seed(T + E)
    z = (torch.randn(T, E, generator=gen) * 2).to(dtype)
    bias = torch.randn(E, generator=gen) * 0.2
    size = E // groups
    bias[torch.rand(E, generator=gen) < 0.5] = off
    bias[:size] = off
    bias[2] = 0.9  # the first group: one expert on (group_best 2: its key is that one's)
    if groups > 1:
        bias[size:2 * size] = off  # a group without any
    else:
        bias[k - 2:] = off  # fewer than k on
    bias[size - 1] = math.inf if T == 97 else bias[size - 1]
    got = L.route(z.cuda(), k, score=score, bias=bias.cuda(), groups=groups, top_groups=top_groups, group_best=group_best)
    some = torch.arange(0, T, 1 + T // 97)
    at, s = _choice(z[some], bias, k, score, groups, top_groups, group_best)
    assert torch.equal(got["indices"][some].cpu().long(), at)
    # exponentials, a sum of up to E of them and two divisions in fp32: (E + 16) half units
    w = s / s.sum(1, keepdim=True)
    assert ((got["weights"][some].double().cpu() - w).abs() <= (E + 16) * 2.0 ** -24 * w).all()
    every = got["indices"][got["indices"] >= 0].long()
    assert torch.equal(got["counts"].long(), torch.bincount(every, minlength=E))


@pytest.mark.parametrize("T", [33, 12301])
@pytest.mark.parametrize("E,k,groups,top_groups,group_best", SWITCHES + [(64, 12, 4, 4, 1), (256, 8, 8, 4, 2)])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("value", [-1e9, -3e38, -2.0 ** 18, -100.0, -64.5, -20.0, 40.0, 1000.0, 1e9])
def test_route_large_biases(L, T, E, k, groups, top_groups, group_best, score, value):
    """Finite biases far from the others: some experts of every group, all of one and all but one of another have one; the logits
    come from a coarse grid, so that choices are contested."""
    gen = torch.Generator().manual_seed(T + E)
    z = (torch.randn(T, E, generator=gen) * 4).round() / 4 + torch.randn(T, E, generator=gen) * 2.0 ** -20
    bias = torch.randn(E, generator=gen) * 0.2
    size = E // groups
    far = torch.rand(E, generator=gen) < 0.3
    far[:size] = True
    far[1] = False
    if groups > 1:
        far[size:2 * size] = True
    else:
        far[k - 2:] = True
    if value > 0:
        far = torch.rand(E, generator=gen) < 0.1
    bias[far] += value
    got = L.route(z.cuda(), k, score=score, bias=bias.cuda(), groups=groups, top_groups=top_groups, group_best=group_best)
    some = torch.arange(0, T, 1 + T // 97)
    at, _ = _choice(z[some], bias, k, score, groups, top_groups, group_best)
    assert torch.equal(got["indices"][some].cpu().long(), at)


def _wide(t):
    return None if t is None else t.double().cpu()


@pytest.mark.parametrize("T,E,k", [(1, 4, 3), (60, 6, 3)])  # each slot by itself; slots ordered by expert
@pytest.mark.parametrize("least", [1e-3, 1e-6])
def test_experts_small_weights(L, T, E, k, least):
    """fp16, routing weights down to `least`: weighted hidden values and dz fall below fp16's normal range, and stay within the bounds
    that say so (an absolute 2^-24 a rounding)."""
    gen = torch.Generator().manual_seed(T)
    D, I = 136, 72
    x, dy = _normal(gen, T, D, dtype=FP16), _normal(gen, T, D, dtype=FP16)
    w1, w2 = _normal(gen, E, 2 * I, D, scale=D ** -0.5, dtype=FP16), _normal(gen, E, D, I, scale=I ** -0.5, dtype=FP16)
    b1, b2 = _normal(gen, E, 2 * I, scale=0.3, dtype=FP16), _normal(gen, E, D, scale=0.3, dtype=FP16)
    at = torch.rand(T, E, generator=gen).topk(k, dim=1).indices.int()
    weights = least ** torch.rand(T, k, generator=gen)
    args = [_wide(x), at, weights.double(), _wide(w1), _wide(w2), _wide(b1), _wide(b2)]
    y = L.experts(x, at.cuda(), weights.cuda(), w1, w2, b1, b2, act="silu", gated=True)
    ref.close(y, *ref.experts(*args, None, "silu", True, FP16), "y")
    got = L.experts_backward(x, at.cuda(), weights.cuda(), w1, w2, dy, b1, b2, act="silu", gated=True)
    for n, (v, bound) in ref.experts_backward(*args, _wide(dy), "silu", True, FP16).items():
        ref.close(got[n], v, ref.rounded(v, bound, FP32) if n == "dweights" else bound, n)


@pytest.mark.parametrize("T,E,k", [(1, 4, 3), (60, 6, 3)])
def test_experts_large_values(L, T, E, k):
    """fp16, hidden values up to the upper end of its range: finite, and within the bounds."""
    gen = torch.Generator().manual_seed(T)
    D, I = 136, 72
    w1 = _normal(gen, E, 2 * I, D, scale=D ** -0.5, dtype=FP16)
    x = torch.randn(T, D, generator=gen)
    at = torch.rand(T, E, generator=gen).topk(k, dim=1).indices.int()
    most = lambda v: max(float(ref.hidden(v.half().double(), _wide(w1[e]), None, "silu", True)[0][(at == e).any(1)].abs().max()) for e in at.unique().tolist())  # noqa: E731
    for _ in range(4):
        x = x * (5e4 / most(x)) ** 0.5
    assert 4e4 < most(x) < 6e4
    x = x.half().cuda()
    w2 = _normal(gen, E, D, I, scale=0.1 * I ** -0.5, dtype=FP16)
    weights = torch.ones(T, k)
    y = L.experts(x, at.cuda(), weights.cuda(), w1, w2, act="silu", gated=True)
    assert y.isfinite().all()
    ref.close(y, *ref.experts(_wide(x), at, weights.double(), _wide(w1), _wide(w2), None, None, None, "silu", True, FP16), "y")


@pytest.mark.parametrize("T", [40, 16400])
@pytest.mark.parametrize("base", [-60.0, -82.0, -87.0, -88.5, -95.0, -104.0, -200.0, -600.0])
@pytest.mark.parametrize("k", [1, 6])
def test_sigmoid_scores_below_fp32(L, T, base, k):
    """Renormalised sigmoid scores of logits far below zero: the ratios count, also where the scores themselves are below fp32's range.
    Exponents of up to 16 apart, rounded to fp32, are off by 16 half units, and the exponentials, sums and divisions by up to 64 more."""
    gen = torch.Generator().manual_seed(3)
    E = 64
    z = (base + torch.randn(T, E, generator=gen) * 2).float()
    z[::5, :3] += 70  # rows with a few scores in range
    got = L.route(z.cuda(), k, score="sigmoid", renorm=True)
    some = torch.arange(0, T, 1 + T // 97)
    at = got["indices"][some].cpu().long()
    x = z[some].double().requires_grad_()
    assert torch.equal(at, x.detach().topk(k, dim=1).indices)
    # sigmoid(x) = exp(x) / (1 + exp(x)), in logarithms
    w = torch.softmax(torch.nn.functional.logsigmoid(x).gather(1, at), 1)
    assert ((got["weights"][some].double().cpu() - w).abs() <= 80 * 2.0 ** -24 * w).all()
    dw = torch.randn(T, k, generator=gen)
    (w * dw[some].double()).sum().backward()
    dz = L.route_backward(z.cuda(), got["indices"], dw.cuda(), score="sigmoid", renorm=True)[some].double().cpu()
    # w (1 - s) (dw - mean): of each factor as above, relative to the largest difference
    spread = (dw[some].double().abs().max(1, keepdim=True).values * 2).expand(-1, E)
    size = torch.zeros_like(dz).scatter_(1, at, w.detach())
    assert ((dz - x.grad).abs() <= 256 * 2.0 ** -24 * size * spread).all()


def _too_much(L):
    """A call that fails for want of memory."""
    from paper_2608_24067_b200.som import SomError
    T, E, k, D, I = 1 << 17, 32, 32, 8192, 8
    assert T * k * D * 6 > torch.cuda.get_device_properties(0).total_memory
    args = (torch.zeros(T, D, dtype=BF16, device="cuda"), torch.zeros(T, k, dtype=torch.int32, device="cuda"), torch.zeros(T, k, device="cuda"),
            torch.zeros(E, 2 * I, D, dtype=BF16, device="cuda"), torch.zeros(E, D, I, dtype=BF16, device="cuda"))
    with pytest.raises(SomError) as e:
        L.experts(*args)
    assert e.value.status == 4 and e.value.cuda_error == 2  # out of memory
    del args, e
    torch.cuda.empty_cache()


def test_workspace_that_cannot_be_had(L):
    """A call whose workspace does not fit the card (4.2 million rows of 8192 in fp32 and 16 bits: 206 GB) says so; neither the handle nor
    what else runs in the process is affected."""
    gen = torch.Generator().manual_seed(2)
    x, w = _normal(gen, 100, 256, dtype=BF16), _normal(gen, 512, 256, dtype=BF16)
    want = L.linear(x, w, act="gelu")
    _too_much(L)
    assert float((torch.ones(8, device="cuda") + 1).sum()) == 16  # (a check of the last CUDA error comes with every launch)
    torch.cuda.synchronize()
    assert torch.equal(L.linear(x, w, act="gelu"), want)
    s = torch.rand(40, 8, generator=gen).topk(4, dim=1)
    y = L.experts(_normal(gen, 40, 64, dtype=BF16), s.indices.int().cuda(), s.values.cuda(), _normal(gen, 8, 64, 64, dtype=BF16), _normal(gen, 8, 64, 32, dtype=BF16))
    assert y.isfinite().all() and L.device_flags() == 0


@pytest.mark.parametrize("T", [40, 16400])
@pytest.mark.parametrize("dtype", [FP32, BF16, FP16])
@pytest.mark.parametrize("k,groups", [(1, 1), (3, 1), (2, 4)])
def test_softmax_masks_of_the_lowest_value(L, T, dtype, k, groups):
    """Logits of the type's lowest value as a mask: such an expert's score is 0 in 64 bits.  Where the bias has only such experts chosen,
    renormalised weights are 0 and not 1 / k, and nothing flows back; beside one that is not masked they weigh 0."""
    gen = torch.Generator().manual_seed(T)
    E = 64
    z = (torch.randn(T, E, generator=gen) * 2).to(dtype)
    low = torch.rand(T, E, generator=gen) < 0.6
    low[:, 7] = False
    z[low] = torch.finfo(dtype).min
    bias = torch.randn(E, generator=gen) * 0.5  # (beyond the scores: it decides)
    opt = dict(score="softmax", groups=groups, top_groups=1, group_best=1)
    got = L.route(z.cuda(), k, bias=bias.cuda(), renorm=True, **opt)
    at = got["indices"].cpu().long()
    x = z.double().requires_grad_()
    q = torch.softmax(x, 1).gather(1, at)
    w = q / q.sum(1, keepdim=True).clamp_min(1e-300)
    masked = low.gather(1, at)
    assert masked.all(1).any() and (masked.any(1) & ~masked.all(1)).any() == (k > 1)
    # (E + 16) half units for exponentials, sums and divisions, 16 for differences of exponents of up to 16
    assert ((got["weights"].double().cpu() - w).abs() <= (E + 32) * 2.0 ** -24 * w).all()
    assert not got["weights"].cpu()[masked].any()
    dw = torch.randn(T, k, generator=gen)
    (w * dw.double()).sum().backward()
    dz = L.route_backward(z.cuda(), got["indices"], dw.cuda(), score="softmax", renorm=True).double().cpu()
    bound = (E + 3 * k + 48) * 2.0 ** -23 * dw.double().abs().max(1, keepdim=True).values
    assert ((dz - x.grad).abs() <= bound + (0 if dtype == FP32 else 2.0 ** -8 * x.grad.abs())).all()
    assert not dz.gather(1, at)[masked].any()


def test_search_after_a_failed_call(L):
    """The error of a call that failed is that call's: the next one, of another handle of the library, does not find it."""
    from paper_2608_24067_b200 import synth
    from paper_2608_24067_b200.som import Som
    V, M = 500, 256
    batch = synth.sample_csr(1000, V, 5.0, 1, device="cuda")
    som = Som(V, M, synth.fill_codebook(V, M, 1, device="cuda"))
    som.norms()
    want, _ = som.bmu(batch.indptr, batch.indices)
    _too_much(L)
    som.norms()
    got, _ = som.bmu(batch.indptr, batch.indices)
    assert torch.equal(got, want)
