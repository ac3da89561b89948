"""Matrices in 4 bits and the linear layer on them against their definitions in 64 bits."""
import pytest
import torch

import train_reference as ref
from train_reference import TYPES

pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)
from paper_2608_24067_b200.layers import Fp4Matrix, Layers  # noqa: E402
from paper_2608_24067_b200.som import SomError  # noqa: E402


@pytest.fixture(scope="module")
def L():
    return Layers()


def scale_bytes(q, D):
    """[rows][blocks] from the order in memory."""
    rows = torch.arange(q.shape[0], device="cuda")[:, None]
    blocks = torch.arange(D // 32, device="cuda")[None]
    return q.scales[ref.scale_at(rows, blocks, D)].long()


def check_matrix(L, x):
    value, code, byte = ref.fp4(x)
    q = L.quantize_fp4(x)
    assert q.shape == tuple(x.shape)
    got = torch.stack([q.codes & 15, q.codes >> 4], 2).view(x.shape).long().cpu()
    lost = (byte == 255).repeat_interleave(32, dim=1)
    assert torch.equal(scale_bytes(q, x.shape[1]).cpu(), byte)
    assert torch.equal(got[~lost], code[~lost])
    for t in TYPES.values():
        v = L.values_fp4(q, dtype=t)
        want = value.to(t)
        assert v.dtype is t and torch.equal(v.isnan().cpu(), lost) and torch.equal(v.cpu()[~lost], want[~lost])
    return q


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("T,D", [(1, 32), (3, 64), (1, 4096), (130, 288), (257, 1024), (33, 2080), (1000, 256)])
def test_sizes(L, T, D, kind):
    gen = torch.Generator(device="cuda").manual_seed(T + D)
    x = torch.randn(T, D, generator=gen, device="cuda") * torch.exp2(torch.randint(-30, 10, (T, D // 32), generator=gen, device="cuda").float()).repeat_interleave(32, 1)
    check_matrix(L, x.to(TYPES[kind]))


def test_every_tie_and_border(L):
    """All halves between two values, on both sides of them, and largest magnitudes around 1.75 times a power of two."""
    half = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    some = torch.cat([half, half * (1 + 2.0 ** -23), half * (1 - 2.0 ** -23)])
    some = torch.cat([some, -some])[:31]
    rows = []
    for power in (-126, -20, 0, 3, 100):
        for top in (4.0, 5.0, 6.0, 7.0, 7.0 * (1 - 2.0 ** -22), 7.99):
            rows.append(torch.cat([some.clamp(-top, top), torch.tensor([top])]) * 2.0 ** power)
    check_matrix(L, torch.stack(rows).cuda())


def test_ends_of_the_range(L):
    x = torch.zeros(8, 64, device="cuda")
    x[0, 3] = 2.0 ** -149
    x[1, 5], x[1, 40] = 2.0 ** -126, 1e-40
    x[2, 0], x[2, 1] = 3.4028234e38, -1e38
    x[3, 7] = float("inf")
    x[4, 33] = float("nan")
    x[5, :32] = -0.0
    x[6, 9], x[6, 10] = -float("inf"), 1.0
    x[7] = 1e-3
    check_matrix(L, x)


def test_rows_apart(L):
    whole = torch.randn(40, 320, device="cuda").bfloat16()
    part = whole[:, 32:288]
    a, b = L.quantize_fp4(part), L.quantize_fp4(part.contiguous())
    assert torch.equal(a.codes, b.codes) and torch.equal(scale_bytes(a, 256), scale_bytes(b, 256))


def test_blocks_beyond_a_row_are_zero_and_rows_beyond_the_last_untouched(L):
    x = torch.randn(5, 288, device="cuda")
    q = L.quantize_fp4(x)
    blocks = torch.arange(9, 16, device="cuda")[None]
    assert not bool(q.scales[ref.scale_at(torch.arange(5, device="cuda")[:, None], blocks, 288)].any())
    scales = torch.full_like(q.scales, 77)
    rc = L._lib.som_fp4_quantize(L._h, 0, 5, 288, x.data_ptr(), 288, q.codes.data_ptr(), scales.data_ptr(), L._stream())
    assert rc == 0
    rest = ref.scale_at(torch.arange(5, 128, device="cuda")[:, None], torch.arange(16, device="cuda")[None], 288)
    assert bool((scales[rest] == 77).all())


# ---- the linear layer --------------------------------------------------------------------------------------------

def layer(T, D, F, kind, gated=False, bias=True, residual=True, seed=0, wild=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[kind]
    new = lambda *s, scale=1.0: (torch.randn(*s, generator=gen, device="cuda") * scale).to(t)  # noqa: E731
    rows = F * (2 if gated else 1)
    x, w = new(T, D), new(rows, D, scale=D ** -0.5)
    if wild:  # blocks of very different sizes
        x = (x.float() * torch.exp2(torch.randint(-6, 4, (T, D // 32), generator=gen, device="cuda").float()).repeat_interleave(32, 1)).to(t)
        w = (w.float() * torch.exp2(torch.randint(-6, 4, (rows, D // 32), generator=gen, device="cuda").float()).repeat_interleave(32, 1)).to(t)
    return x, w, new(rows, scale=0.1) if bias else None, new(T, F) if residual else None


def check_layer(L, x, w, bias, residual, act="none", gated=False, out=None):
    q = L.quantize_fp4(w)
    y = L.linear_fp4(x, q, bias, residual, act=act, gated=gated, out=out)
    want, tol = ref.fp4_linear(x, L.values_fp4(q, torch.float32), bias, residual, act, gated)
    bad = ~((y.double() - want).abs() <= tol)
    assert not bool(bad.any()), "%d of %d, first at %s, the worst %.3g of what is allowed" % (
        int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), float(((y.double() - want).abs() / tol).max()))
    assert L.device_flags() == 0
    return y


SIZES = [(1, 32, 8), (1, 4096, 1024), (2, 256, 520), (3, 288, 264), (5, 512, 128), (8, 2080, 96), (16, 1024, 512), (31, 544, 776), (65, 2048, 4104), (128, 256, 128), (129, 320, 136), (300, 1056, 1000),
         (513, 768, 2056), (1000, 512, 640)]


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("T,D,F", SIZES)
def test_linear(L, T, D, F, kind):
    check_layer(L, *layer(T, D, F, kind, seed=T, wild=True))


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("T,D,F", [(1, 512, 256), (4, 320, 72), (40, 512, 256), (200, 288, 264), (700, 1024, 512), (530, 96, 1000)])
def test_activations_and_gates(L, T, D, F, act):
    for gated in (False, True):
        for bias, residual in ((True, True), (False, False)):
            check_layer(L, *layer(T, D, F, "bf16", gated, bias, residual), act=act, gated=gated)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("T", [1, 2, 3, 4])
@pytest.mark.parametrize("D,F,gated", [(32, 8, False), (96, 136, False), (4096, 640, True), (1056, 1000, False), (7200, 264, False), (64, 4096, False), (2048, 128, True), (20000, 8, False), (544, 72, True)])
def test_a_few_rows(L, T, D, F, gated, kind):
    """One row to four: one step of 1024 columns and several, columns shared by warps, features that end inside 128."""
    check_layer(L, *layer(T, D, F, kind, gated, seed=D, wild=True), act="silu", gated=gated)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("T,D,F,gated", [(1500, 1056, 2056, False), (2900, 544, 3200, False), (1300, 512, 1024, True), (1409, 288, 1000, True), (5000, 256, 640, False), (2200, 2080, 2304, True)])
def test_pairs_of_blocks(L, T, D, F, gated, kind):
    """Tiles of 256 x 256, one to several rounds of them, with rows and columns that end inside a tile."""
    check_layer(L, *layer(T, D, F, kind, gated, seed=T, wild=True), act="gelu" if T % 2 else "none", gated=gated)


@pytest.mark.parametrize("T", [1, 7, 140, 6200])
def test_no_column_of_the_weights_is_mixed_up(L, T):
    """Weights and rows with one block that counts: every block of every row meets its own scale."""
    D, F = 1088, 392
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.zeros(T, D, device="cuda", dtype=torch.bfloat16)
    at = torch.randint(0, D, (T,), generator=gen, device="cuda")
    x[torch.arange(T, device="cuda"), at] = torch.exp2(torch.randint(-8, 8, (T,), generator=gen, device="cuda").float()).bfloat16()
    w = (torch.randint(1, 4, (F, D), generator=gen, device="cuda") * torch.exp2(torch.randint(-8, 8, (F, D // 32), generator=gen, device="cuda").float()).repeat_interleave(32, 1)).bfloat16()
    q = L.quantize_fp4(w)
    y = L.linear_fp4(x, q)
    want = x.double() @ L.values_fp4(q, torch.float32).double().t()  # a single product each: exact but for the last rounding
    assert torch.equal(y, want.to(torch.bfloat16))


@pytest.mark.parametrize("T", [1, 33, 300, 9700])
def test_nan_stays_in_its_row(L, T):
    x, w, b, r = layer(T, 512, 256, "bf16")
    q = L.quantize_fp4(w)
    clean = L.linear_fp4(x, q, b, r)
    w[77, 100] = float("nan")
    x[T // 2, 300] = float("inf")
    y = L.linear_fp4(x, L.quantize_fp4(w), b, r)
    bad = torch.zeros_like(y, dtype=torch.bool)
    bad[T // 2], bad[:, 77] = True, True
    assert bool(y[bad].isnan().all()) and torch.equal(y[~bad], clean[~bad])


@pytest.mark.parametrize("T", [1, 40, 400])
def test_only_the_rows_are_written(L, T):
    x, w, b, r = layer(T, 256, 264, "bf16")
    whole = torch.full((T, 304), 9.0, device="cuda", dtype=torch.bfloat16)
    y = check_layer(L, x, w, b, r, act="silu", out=whole[:, 16:280])
    assert bool((whole[:, :16] == 9).all()) and bool((whole[:, 280:] == 9).all()) and torch.equal(y, whole[:, 16:280])


@pytest.mark.parametrize("T,D,F", [(1, 2048, 2048), (50, 2048, 512), (600, 1024, 1024), (4000, 512, 2048)])
def test_same_bits_every_time_and_in_a_graph(L, T, D, F):
    x, w, b, r = layer(T, D, F, "bf16")
    q = L.quantize_fp4(w)
    first = L.linear_fp4(x, q, b, r, act="gelu")
    for _ in range(5):
        assert torch.equal(first, L.linear_fp4(x, q, b, r, act="gelu"))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = L.linear_fp4(x, q, b, r, act="gelu")
    again.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, again)


def test_offsets_beyond_32_bits(L):
    """Rows whose elements lie beyond 2^31 get what they get by themselves, in a product of the same tiles."""
    T, D, F, last = 1100000, 2048, 64, 40000
    x = torch.zeros(T, D, device="cuda", dtype=torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(2)
    x[-last:] = torch.randn(last, D, generator=gen, device="cuda").bfloat16()
    part = x[-last:].clone()
    a, b = L.quantize_fp4(x), L.quantize_fp4(part)
    assert torch.equal(a.codes[-last:], b.codes)
    values = L.values_fp4(a)
    assert torch.equal(values[-last:], L.values_fp4(b)) and not bool(values[:-last].any())
    del values
    w = L.quantize_fp4(torch.randn(F, D, generator=gen, device="cuda").bfloat16())
    y = L.linear_fp4(x, w)
    assert torch.equal(y[-last:], L.linear_fp4(part, w)) and not bool(y[:-last].any()) and L.device_flags() == 0


def test_strided_operands(L):
    x, w, b, r = layer(70, 512, 256, "fp16")
    wide, far = torch.zeros(70, 640, device="cuda", dtype=torch.float16), torch.zeros(70, 512, device="cuda", dtype=torch.float16)
    wide[:, 64:576], far[:, 8:264] = x, r
    q = L.quantize_fp4(w)
    assert torch.equal(L.linear_fp4(wide[:, 64:576], q, b, far[:, 8:264]), L.linear_fp4(x, q, b, r))


def test_another_stream(L):
    x, w, b, r = layer(70, 512, 256, "bf16")
    want = L.linear_fp4(x, L.quantize_fp4(w), b, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q = L.quantize_fp4(w, stream=side)
    got = L.linear_fp4(x, q, b, r, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_no_rows(L):
    x, w, _, _ = layer(4, 64, 32, "bf16")
    assert L.linear_fp4(x[:0], L.quantize_fp4(w)).shape == (0, 32)
    assert L.values_fp4(L.quantize_fp4(x[:0])).shape == (0, 64)


def test_refusals(L):
    x, w, b, r = layer(4, 64, 32, "bf16")
    q = L.quantize_fp4(w)
    for bad in (lambda: L.quantize_fp4(x[:, :40]), lambda: L.quantize_fp4(x.int()), lambda: L.quantize_fp4(x[0]), lambda: L.quantize_fp4(x.t()), lambda: L.values_fp4(w),
                lambda: L.values_fp4(q, torch.float64), lambda: L.linear_fp4(x, w), lambda: L.linear_fp4(x.float(), q), lambda: L.linear_fp4(x[:, :32], q), lambda: L.linear_fp4(x, q, b[:5]),
                lambda: L.linear_fp4(x, q, b, r[:2]), lambda: L.linear_fp4(x, q, act="tanh"), lambda: Fp4Matrix(q.codes.int(), q.scales), lambda: L.linear_fp4(x, Fp4Matrix(q.codes, q.scales[:100])),
                lambda: L.quantize_fp4(x.cpu()), lambda: L.linear_fp4(x, Fp4Matrix(q.codes.cpu(), q.scales.cpu()))):
        with pytest.raises((TypeError, ValueError)):
            bad()
    whole = torch.zeros(4, 72, device="cuda", dtype=torch.bfloat16)
    for bad in (lambda: L.quantize_fp4(whole[:, 4:68]), lambda: L.linear_fp4(whole[:, 4:68], q), lambda: L.linear_fp4(x, L.quantize_fp4(x.repeat(3, 1)[:12]), gated=True)):
        with pytest.raises(SomError):  # rows off 16 bytes; 6 outputs
            bad()
