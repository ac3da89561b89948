"""AdamW writes its parameters' memory by address: a parameter or copy whose memory was exchanged after the optimiser was made is refused,
before anything reaches the library (the old address may be another tensor's by then)."""
import pytest
import torch

from paper_2608_24067_b200 import layers
from test_layers_cpu import BF16, _handle, _On, _Refused


def _on(*shape, t=torch.float32):
    return torch.zeros(*shape, dtype=t).as_subclass(_On)


EXCHANGES = {
    "other memory": lambda p: setattr(p, "data", torch.zeros(p.shape, dtype=p.dtype)),
    "a part of its memory": lambda p: setattr(p, "data", p.data[:2]),
    "other order": lambda p: setattr(p, "data", p.data.t()),
    "other type": lambda p: setattr(p, "data", p.data.view(torch.int32 if p.dtype is torch.float32 else torch.float16)),
    "set_": lambda p: p.set_(torch.zeros(p.shape, dtype=p.dtype)),
    "resize_": lambda p: p.resize_(1000, 1000),
    "empty": lambda p: setattr(p, "data", torch.zeros(0, dtype=p.dtype)),
}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("which", ["a parameter", "a copy", "a 16-bit parameter"])
@pytest.mark.parametrize("how", EXCHANGES)
def test_exchanged_memory_is_refused(how, which, bits):
    h = _handle()
    p, q, r, c = _on(4, 4), _on(8, 8), _on(4, 4, t=BF16), _on(8, 8, t=BF16)
    opt = layers.AdamW(h, [p, q, r], copies=[None, c, None], bits=bits)
    grads = [_on(4, 4), _on(8, 8), _on(4, 4, t=BF16)]
    with pytest.raises(_Refused):  # all in its place: the call goes through to the library
        opt.step(grads)
    EXCHANGES[how]({"a parameter": q, "a copy": c, "a 16-bit parameter": r}[which])
    with pytest.raises(ValueError):
        opt.step(grads)
    with pytest.raises(ValueError):
        opt.step([g.reshape(x.shape) if g.numel() == x.numel() else g for g, x in zip(grads, (p, q, r))])
    assert opt.steps == 0


def test_values_written_in_place_are_not_an_exchange():
    h = _handle()
    p = _on(4, 4)
    opt = layers.AdamW(h, [p])
    p.copy_(torch.ones(4, 4))
    p.data.mul_(2)
    with pytest.raises(_Refused):
        opt.step([_on(4, 4)])
    p.data = p.data.view(4, 4)
    with pytest.raises(_Refused):
        opt.step([_on(4, 4)])


def test_what_it_writes_cannot_be_exchanged():
    opt = layers.AdamW(_handle(), [_on(4), _on(4)], copies=[_on(4, t=BF16), None])
    for some in (opt.params, opt.copies):
        with pytest.raises(TypeError):
            some[0] = _on(4)
