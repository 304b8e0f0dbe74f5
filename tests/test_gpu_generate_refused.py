"""A step of generating that is refused, whoever refuses it, leaves the sequences and the free pages as they were."""
import pytest
import torch

import paper_2105_00053_amd as pn
from paper_2105_00053_amd import lm_step
from test_gpu_lm_step import make

pytestmark = pytest.mark.gpu


def state(cache):
    return list(cache.free), {name: (list(pages), n) for name, (pages, n) in cache.held.items()}


def refused(cache, call):
    before = state(cache)
    with pytest.raises(pn.PositError):
        call()
    assert state(cache) == before


def test_heads_that_pages_do_not_take():
    net, _ = make(3, d=12)
    cache = lm_step.PagedDecoder(net, pages=4, page=16)
    refused(cache, lambda: cache.step({"a": [1, 2, 3]}))
    refused(cache, lambda: cache.sample({"a": [1]}, torch.zeros(1, device="cuda")))
    assert cache.length("a") == 0


def test_more_rows_than_attention_takes_and_wrong_draws():
    net, g = make(5, rotated=16, head_norms=True)
    text = torch.randint(0, 67, (640,), generator=g).tolist()
    cache, plain = (lm_step.PagedDecoder(net, pages=14, page=64) for _ in range(2))
    u = torch.full((2,), 0.5, device="cuda")
    for c in (cache, plain):
        c.step({"a": text[:20], "b": text[:70]})
    refused(cache, lambda: cache.step({"b": text[70:73], "c": text[:600]}, most_rows=10 ** 6))   # 600 positions of two heads
    refused(cache, lambda: cache.step({"c": text[:600], "d": text}))                            # too few pages
    refused(cache, lambda: cache.sample({"a": [3]}, u))                                         # two numbers for one row
    refused(cache, lambda: cache.sample({"a": [3], "c": text[:100]}, u, top_k=u))
    # and goes on as if they had not been asked for
    for new in ({"b": text[70:73], "c": text[:600]}, {"a": [3], "c": [7]}):
        assert torch.equal(lm_step._movable(cache.step(new)), lm_step._movable(plain.step(new)))
    assert all(torch.equal(s, t) for s, t in zip(cache.sample({"c": [1], "b": [2]}, u), plain.sample({"c": [1], "b": [2]}, u)))
    assert state(cache) == state(plain)
