"""Parameters of a module whose memory a module's own calls exchange: refused by the next step, nothing is changed, and a new optimiser goes on."""
import pytest
import torch

pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)
from paper_2608_24067_b200.layers import AdamW, Layers  # noqa: E402


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("exchange", [lambda m: m.half(), lambda m: m.bfloat16().float(), lambda m: [setattr(p, "data", p.data.clone()) for p in m.parameters()]])
def test_a_module_s_exchanged_parameters(bits, exchange):
    L = Layers()
    module = torch.nn.Linear(40, 30).cuda()
    grads = [torch.ones_like(p) for p in module.parameters()]
    opt = AdamW(L, module.parameters(), bits=bits)
    opt.step(grads)
    m, v = ([x.clone() for x in some] for some in opt.moments())
    old = [p.data for p in module.parameters()]  # (keeps the old memory)
    exchange(module)
    kept = [(p.clone(), q.clone()) for p, q in zip(module.parameters(), old)]
    with pytest.raises(ValueError):
        opt.step(grads)
    assert opt.steps == 1 and all(torch.equal(p, a) and torch.equal(q, b) for (a, b), p, q in zip(kept, module.parameters(), old))
    assert all(torch.equal(a, b) for a, b in zip((*m, *v), (*opt.moments()[0], *opt.moments()[1])))
    again = AdamW(L, module.parameters(), bits=bits)
    again.load(*opt.state(), steps=opt.steps)
    again.step([g.to(p.dtype) for g, p in zip(grads, module.parameters())])
    assert again.steps == 2 and all(bool((p != a).any()) for p, (a, _) in zip(module.parameters(), kept))
