"""The dense operators' C entries without a GPU: null handles and arguments are refused before anything touches a device."""
import ctypes
import os
import re

import pytest
import torch

from paper_2608_24067_b200 import som


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
