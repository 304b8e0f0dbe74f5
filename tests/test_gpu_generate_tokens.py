"""Tokens that are none of the table's are refused on the host, before anything is launched: the draw's -1 among them."""
import pytest
import torch

import paper_2105_00053_amd as pn
from paper_2105_00053_amd import lm_step
from test_gpu_lm_step import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [[-1], [67], [0, 66, -67], [5, 2 ** 31 - 1], [1 << 40]])
def test_tokens_outside_the_table(tokens):
    net, _ = make(3)
    cache = lm_step.PagedDecoder(net, pages=4, page=16)
    cache.step({"a": [0, 66]})
    with pytest.raises(pn.PositError):
        cache.step({"a": [1], "b": tokens})
    with pytest.raises(pn.PositError):
        cache.sample({"a": tokens}, torch.zeros(1, device="cuda"))
    assert cache.length("a") == 2 and cache.length("b") == 0 and len(cache.free) == 3
    cache.step({"a": [66], "b": [0]})
    torch.cuda.synchronize()
