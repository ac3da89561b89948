"""The dense operators' C entries without a GPU: null handles and arguments are refused before anything touches a device."""
import ctypes
import os
import re

import pytest
import torch

from paper_2608_24067_b200 import layers, som


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


def _source(name):
    return open(os.path.join(os.path.dirname(som.__file__), "csrc", name)).read()


def test_epilogue_gives_up_as_one():
    """The epilogue's warps meet at a hardware barrier in every tile, so they have to leave together: whether a wait ran out is read
    from a word that only the waiting lane writes, before the barrier, never from the flag that other warps may raise at any time."""
    text = re.sub(r"//[^\n]*", "", _source("layers_product.cu"))
    loop = text[text.index("Stager<out_buffers(MODE)> s{"):]
    loop = loop[:loop.index("if (warp >= 2 && lane == 0) store_wait_all()")]
    assert loop.count("bar.sync 1") == 1
    before, after = loop.split("bar.sync 1")
    word = re.search(r"(\w+)\[n_acc & 1\] = bar_wait\(&acc_full\[buf\],", before)
    assert word and "*gave_up" not in loop
    assert re.match(r'[^\n]*"memory"\);\s*if \(!%s\[n_acc & 1\]\) break;' % word.group(1), after)
    # (the other word is in use until every warp has passed the next tile's barrier: two take turns)
    assert re.search(r"__shared__ int[^;]*\b%s\[2\]" % word.group(1), text)
    assert len(re.findall(r"\b%s\[" % word.group(1), loop)) == 2  # written once, read once


def test_pair_waits_at_the_scope_it_arrives_at():
    """A pair's accumulator is freed by arrivals from both blocks: they are made, and have to be waited for, at cluster scope."""
    ptx, product = _source("layers_ptx.cuh"), _source("layers_product.cu")
    assert "mbarrier.arrive.relaxed.cluster.shared::cluster.b64" in ptx
    assert "mbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64" in ptx
    waits = re.findall(r"bar_wait(<\w+>)?\(&acc_empty", product)
    assert waits and set(waits) == {"<PAIRED>"}


class _On(torch.Tensor):
    """A CPU tensor that says that it lies on GPU `index`."""

    index = 0
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.index))
    get_device = lambda self: self.index  # noqa: E731


class _Refused(AssertionError):
    pass


class _Library:
    """Stands for the compiled library: no call may get this far."""

    def __getattr__(self, name):
        def call(*a):
            raise _Refused(name)
        return call


def _handle():
    h = layers.Layers.__new__(layers.Layers)
    h._lib, h._h, h.device = _Library(), ctypes.c_void_p(), torch.device("cuda", 0)
    h._stream = lambda stream=None: 0
    return h


T, E, K, D, I = 4, 3, 2, 64, 16
BF16 = torch.bfloat16
TENSORS = {
    "linear": {"x": ((T, D), BF16), "weight": ((32, D), BF16), "bias": ((32,), BF16), "residual": ((T, 32), BF16), "out": ((T, 32), BF16)},
    "linear_backward": {"x": ((T, D), BF16), "weight": ((32, D), BF16), "dy": ((T, 32), BF16), "bias": ((32,), BF16)},
    "route": {"logits": ((T, E), torch.float32), "bias": ((E,), torch.float32)},
    "route_backward": {"logits": ((T, E), torch.float32), "indices": ((T, K), torch.int32), "dweights": ((T, K), torch.float32)},
    "experts": {"x": ((T, D), BF16), "indices": ((T, K), torch.int32), "weights": ((T, K), torch.float32), "w1": ((E, 2 * I, D), BF16),
                "w2": ((E, D, I), BF16), "b1": ((E, 2 * I), BF16), "b2": ((E, D), BF16), "residual": ((T, D), BF16), "out": ((T, D), BF16)},
    "experts_backward": {"x": ((T, D), BF16), "indices": ((T, K), torch.int32), "weights": ((T, K), torch.float32), "w1": ((E, 2 * I, D), BF16),
                         "w2": ((E, D, I), BF16), "dy": ((T, D), BF16), "b1": ((E, 2 * I), BF16), "b2": ((E, D), BF16)},
}


def _call(name, elsewhere=None, where=1):
    args = {n: torch.zeros(shape, dtype=dtype).as_subclass(_On) for n, (shape, dtype) in TENSORS[name].items()}
    if elsewhere:
        shape, dtype = TENSORS[name][elsewhere]
        args[elsewhere] = torch.zeros(shape, dtype=dtype)  # where < 0: on the host
        if where >= 0:
            args[elsewhere] = args[elsewhere].as_subclass(type("_Other", (_On,), {"index": where}))
    return getattr(_handle(), name)(**args, **({"k": 2} if name == "route" else {}))


@pytest.mark.parametrize("name", TENSORS)
def test_tensors_of_another_device_are_refused(name):
    """Every tensor of a call has to lie on the handle's device: the address of one that does not would be an illegal access."""
    with pytest.raises(_Refused):  # all on the handle's device: the call goes through to the library
        _call(name)
    for n in TENSORS[name]:
        with pytest.raises(ValueError):
            _call(name, n, 1)
        with pytest.raises((TypeError, ValueError)):
            _call(name, n, -1)


@pytest.mark.parametrize("name", TENSORS)
def test_memory_follows_the_stream(name, monkeypatch):
    """With `stream=` the outputs are that stream's memory (another stream may still have work in memory of its own that was
    freed), and what the call is given and returns is not handed out again while either stream uses it."""
    import contextlib
    now, log = ["main"], []

    class Stream:
        def __init__(self, name):
            self.name, self.cuda_stream, self.device = name, len(name), torch.device("cuda", 0)

    main, side = Stream("main"), Stream("side")

    @contextlib.contextmanager
    def as_current(stream):
        before, now[0] = now[0], stream.name
        yield
        now[0] = before

    monkeypatch.setattr(torch.cuda, "stream", as_current)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: {"main": main, "side": side}[now[0]])

    class Seen(_On):
        def new_empty(self, *a, **kw):
            log.append(("made", now[0]))
            return super().new_empty(*a, **kw).as_subclass(Seen)

        def record_stream(self, stream):
            log.append((self.what if hasattr(self, "what") else "output", stream.name))

    h = _handle()
    h._lib = type("Library", (), {"__getattr__": lambda self, n: lambda *a: log.append(("called", now[0])) or 0})()
    args = {n: torch.zeros(shape, dtype=dtype).as_subclass(Seen) for n, (shape, dtype) in TENSORS[name].items() if n != "out"}
    for n in args:
        args[n].what = n
    kw = {"k": 2} if name == "route" else {}
    getattr(h, name)(**args, **kw)
    assert {w for what, w in log if what in ("made", "called")} == {"main"} and not any(what in args for what, _ in log)
    log.clear()
    out = getattr(h, name)(**args, **kw, stream=side)
    count = len(out) if isinstance(out, dict) else 1
    assert [w for what, w in log if what in ("made", "called")] == ["side"] * (count + 1)
    assert sorted(what for what, w in log if what in args and w == "side") == sorted(args)
    assert log.count(("output", "main")) == count
    other = Stream("far")
    other.device = torch.device("cuda", 1)
    with pytest.raises(ValueError):
        getattr(h, name)(**args, **kw, stream=other)


def test_rounds_without_a_handle():
    assert som.load_library().som_layers_rounds(None, 0, 0) == -1
