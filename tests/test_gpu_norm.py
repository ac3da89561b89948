"""Layer norm and its gradient against their definitions in 64 bits."""
import pytest
import torch

import train_reference as ref
from train_reference import TYPES

pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)
from paper_2608_24067_b200.layers import Layers  # noqa: E402
from paper_2608_24067_b200.som import SomError  # noqa: E402


@pytest.fixture(scope="module")
def L():
    return Layers()


def matrix(gen, T, D, t, apart=0, shift=0, scale=1.0, offset=0.0):
    """[T, D] whose rows lie D + apart elements from each other and start `shift` elements behind an aligned address."""
    v = (torch.randn(T, D, generator=gen, device="cuda") * scale + offset).to(t)
    if not apart and not shift:
        return v
    whole = torch.full((T * (D + apart) + shift,), 7.0, device="cuda", dtype=t)
    part = whole[shift:].view(T, D + apart)[:, :D]
    part.copy_(v)
    return part


def inputs(T, D, kind, weights="same", residual=True, affine=True, apart=0, shift=0, offset=0.5, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[kind]
    wt = t if weights == "same" else torch.float32
    x = matrix(gen, T, D, t, apart, shift, offset=offset)
    r = matrix(gen, T, D, t, apart, shift) if residual else None
    w = (1 + 0.2 * torch.randn(D, generator=gen, device="cuda")).to(wt) if affine else None
    b = (0.1 * torch.randn(D, generator=gen, device="cuda")).to(wt) if affine else None
    dy = matrix(gen, T, D, t, apart, shift)
    return x, r, w, b, dy


def near(got, want, tol, name):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), "%s: %d of %d, the worst by %.3g of what is allowed" % (name, int(bad.sum()), bad.numel(), float(((got.double() - want).abs() / tol).max()))


def check(L, x, r, w, b, dy, eps=1e-5):
    out = L.norm(x, w, b, r, eps=eps)
    y, total = (out["y"], out["sum"]) if r is not None else (out, x)
    want, h, tol = ref.norm(x, w, b, r, eps)
    assert y.shape == x.shape and y.dtype is x.dtype
    if r is not None:
        assert torch.equal(total, h.to(x.dtype))
    near(y, want, tol, "y")
    for dsum in (None, r):
        got = L.norm_backward(total, w, dy, b, dsum, eps=eps)
        want, tol = ref.norm_backward(total, w, dy, dsum, eps)
        near(got["dx"], want["dx"], tol["dx"], "dx")
        assert set(got) == {"dx"} | ({"dweight"} if w is not None else set()) | ({"dbias"} if b is not None else set())
        for n in set(got) - {"dx"}:
            assert got[n].dtype is w.dtype
            rel, least = ref.half_step(w.dtype)
            near(got[n], want[n], tol[n] + rel * want[n].abs() + least, n)


SIZES = [(1, 1), (1, 8), (3, 7), (1, 4096), (2, 33), (5, 1000), (130, 256), (77, 2048), (19, 8192), (3, 8200), (2, 20001), (1500, 64), (700, 1024), (333, 4104), (64, 5120)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("T,D", SIZES)
def test_sizes(L, T, D, kind):
    check(L, *inputs(T, D, kind, seed=T + D))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("T,D,apart,shift", [(5, 1000, 24, 8), (5, 1000, 3, 0), (4, 512, 0, 1), (9, 2048, 8, 4), (3, 31, 2, 5)])
def test_strides_and_alignment(L, T, D, apart, shift, kind):
    check(L, *inputs(T, D, kind, apart=apart, shift=shift))


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("residual,affine", [(False, True), (True, False), (False, False)])
def test_parts(L, residual, affine, kind):
    x, r, w, b, dy = inputs(50, 768, kind, "fp32", residual, affine)
    check(L, x, r, w, b, dy)
    if affine:
        check(L, x, r, w, None, dy)
        out = L.norm(x, None, b)
        near(out, *[v for i, v in enumerate(ref.norm(x, None, b, None, 1e-5)) if i != 1], "bias alone")


@pytest.mark.parametrize("D", [257, 2048, 9000])
def test_rows_far_from_zero(L, D):
    """The variance is that of the differences: a row around 1000 keeps it.  (Any single-pass formula loses all digits here.)"""
    x, _, w, b, dy = inputs(7, D, "fp32", residual=False, offset=1000.0)
    check(L, x, None, w, b, dy)


@pytest.mark.parametrize("D", [64, 1000, 4096])
def test_constant_rows(L, D):
    x = torch.full((3, D), 2.5, device="cuda", dtype=torch.bfloat16)
    w, b = torch.ones(D, device="cuda"), torch.full((D,), 0.25, device="cuda")
    assert torch.equal(L.norm(x, w, b), torch.full_like(x, 0.25))  # the sum of equal values that fp32 holds is exact: nothing is left
    dy = torch.ones_like(x)
    got = L.norm_backward(x, w, dy, b)
    assert torch.equal(got["dx"], torch.zeros_like(x)) and torch.equal(got["dweight"], torch.zeros(D, device="cuda")) and torch.equal(got["dbias"], torch.full((D,), 3.0, device="cuda"))


@pytest.mark.parametrize("D", [512, 333])
def test_sum_without_a_residual_is_x(L, D):
    x, _, w, b, _ = inputs(5, D, "fp16", residual=False)
    total, y = torch.zeros_like(x), torch.zeros_like(x)
    rc = L._lib.som_norm(L._h, 1, 5, D, x.data_ptr(), D, w.data_ptr(), b.data_ptr(), 1, None, 0, 1e-5, total.data_ptr(), D, y.data_ptr(), D, L._stream())
    assert rc == 0 and torch.equal(total, x) and torch.equal(y, L.norm(x, w, b))


def test_infinities_and_nan_stay_in_their_rows(L):
    x, r, w, b, dy = inputs(6, 640, "bf16", residual=False)
    clean, back = L.norm(x, w, b), L.norm_backward(x, w, dy, b)["dx"]
    x[2, 17], x[4, 600] = float("inf"), float("nan")
    y, dx = L.norm(x, w, b), L.norm_backward(x, w, dy, b)["dx"]
    keep = [0, 1, 3, 5]
    assert torch.equal(y[keep], clean[keep]) and torch.equal(dx[keep], back[keep])
    assert not bool(torch.isfinite(y[[2, 4]]).any()) and not bool(torch.isfinite(dx[[2, 4]]).any())


def test_no_rows(L):
    x, _, w, b, dy = inputs(0, 96, "bf16", residual=False)
    assert L.norm(x, w, b).shape == (0, 96)
    got = L.norm_backward(x, w, dy, b)
    assert got["dx"].shape == (0, 96) and not bool(got["dweight"].any()) and not bool(got["dbias"].any())


@pytest.mark.parametrize("kind", TYPES)
def test_only_the_rows_are_written(L, kind):
    x, r, w, b, _ = inputs(5, 200, kind)
    whole = torch.full((5, 232), 9.0, device="cuda", dtype=x.dtype)
    out = L.norm(x, w, b, out=whole[:, 16:216])
    assert bool((whole[:, :16] == 9).all()) and bool((whole[:, 216:] == 9).all())
    assert torch.equal(out, L.norm(x, w, b))


@pytest.mark.parametrize("T,D", [(3000, 2048), (3000, 1001), (9, 4096)])
def test_same_bits_every_time_and_in_a_graph(L, T, D):
    x, r, w, b, dy = inputs(T, D, "bf16")
    first, back = L.norm(x, w, b, r), L.norm_backward(x, w, dy, b, r)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again, back2 = L.norm(x, w, b, r), L.norm_backward(x, w, dy, b, r)
    for v in (*again.values(), *back2.values()):
        v.fill_(1.0)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(first[n], again[n]) for n in first) and all(torch.equal(back[n], back2[n]) for n in back)


def test_another_stream(L):
    x, r, w, b, dy = inputs(100, 512, "fp16")
    want = L.norm(x, w, b, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = L.norm(x, w, b, r, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got["y"], want["y"]) and torch.equal(got["sum"], want["sum"])


def test_offsets_beyond_32_bits(L):
    """Rows whose elements lie beyond 2^31 get what they get by themselves."""
    T, D, last = 1100000, 2048, 333
    x = torch.zeros(T, D, device="cuda", dtype=torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(2)
    x[-last:] = torch.randn(last, D, generator=gen, device="cuda").bfloat16()
    w, b = torch.randn(D, generator=gen, device="cuda").bfloat16(), torch.randn(D, generator=gen, device="cuda").bfloat16()
    y, alone = L.norm(x, w, b, x), L.norm(x[-last:].clone(), w, b, x[-last:].clone())
    assert torch.equal(y["y"][-last:], alone["y"]) and torch.equal(y["sum"][-last:], alone["sum"])
    del y
    dy = torch.zeros_like(x)
    dy[-last:] = torch.randn(last, D, generator=gen, device="cuda").bfloat16()
    got, alone = L.norm_backward(x, w, dy, b), L.norm_backward(x[-last:].clone(), w, dy[-last:].clone(), b)
    assert torch.equal(got["dx"][-last:], alone["dx"]) and not bool(got["dx"][:-last].any())
    for n in ("dweight", "dbias"):  # the same terms in other parts: sums of 333 of size 1 in fp32, rounded to bf16
        off = (got[n].float() - alone[n].float()).abs()
        assert bool((off <= 2.0 ** -7 * alone[n].float().abs() + 333 * 2.0 ** -18).all())


def test_against_differences(L):
    """The gradient against (f(x + h) - f(x - h)) / 2 h of the forward call in fp32, f = sum(dy y), along random directions."""
    x, _, w, b, dy = inputs(4, 300, "fp32", residual=False, seed=5)
    got = L.norm_backward(x, w, dy, b)
    gen = torch.Generator(device="cuda").manual_seed(6)
    f = lambda x, w, b: float((L.norm(x, w, b).double() * dy.double()).sum())  # noqa: E731
    h = 2.0 ** -6
    # y of size 1 is off by some 2^-22; the sum of 1200 such errors, randomly signed, by 35 2^-22, over 2 h: 3e-4.  The third derivative's part
    # is h^2 / 6 of the direction's cube over rows of 300: below 1e-4 of the gradient's size (30)
    for n, grad in (("x", got["dx"]), ("w", got["dweight"]), ("b", got["dbias"])):
        v = {"x": x, "w": w, "b": b}
        d = torch.randn(v[n].shape, generator=gen, device="cuda")
        up, down = dict(v), dict(v)
        up[n], down[n] = v[n] + h * d, v[n] - h * d
        slope = (f(**up) - f(**down)) / (2 * h)
        assert abs(slope - float((grad.double() * d.double()).sum())) < 0.02


def test_refusals(L):
    x, r, w, b, dy = inputs(4, 64, "bf16")
    for bad in (lambda: L.norm(x, w[:32], b), lambda: L.norm(x, w, b.float()), lambda: L.norm(x.int(), w, b), lambda: L.norm(x[0], w, b), lambda: L.norm(x, w, b, r[:2]),
                lambda: L.norm(x, w.half(), b.half()), lambda: L.norm(x.t(), None, None), lambda: L.norm_backward(x, w, dy[:, :32], b), lambda: L.norm(x.cpu(), w, b),
                lambda: L.norm_backward(x, w, dy.float(), b)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    for eps in (-1.0, float("nan")):
        with pytest.raises(SomError):
            L.norm(x, w, b, eps=eps)
    with pytest.raises(SomError):
        L.norm(torch.empty(4, 0, device="cuda", dtype=torch.bfloat16))
