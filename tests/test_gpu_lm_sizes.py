"""Sizes at the ends of what the language-model operators accept."""
import pytest
import torch

import paper_2105_00053_amd as pn
from test_gpu_lm_attention import _inputs

pytestmark = pytest.mark.gpu

MOST = 2 ** 63 - 1


@pytest.mark.parametrize("b,lq,lk,hq,hkv,d", [(4, 1, 4096, 16, 4, 64), (2, 3, 2500, 4, 1, 40), (1, 150, 150, 4, 2, 64), (1, 70, 333, 2, 1, 128)])
def test_windows_and_sinks_beyond_the_cache(b, lq, lk, hq, hkv, d):
    """A window that no position reaches back to the start of is none, sinks beyond the last key are all keys: bit for bit the same result."""
    _, q, k, v, do = _inputs(b, lq, lk, hq, hkv, d, "bf16", "p8_1", 41)
    lens = torch.tensor([lk - 19 * i for i in range(b)], dtype=torch.int32, device="cuda")

    def run(window, sinks):
        how = {"window": window, "sinks": sinks, "lens": lens}
        o, lse, copy = pn.posit_attention_fwd(q, k, v, "bf16", "p8_1", "p8_1", fcopy="f32", **how)
        return (o, lse, copy) + tuple(pn.posit_attention_bwd(do, q, k, v, copy, lse, "bf16", "bf16", "p8_1", "f32", "bf16", **how))

    want = run(0, 0)
    for window, sinks in ((lk, 0), (MOST, 0), (MOST, MOST), (2 ** 31, 4), (0, MOST)):
        assert all(torch.equal(x, y) for x, y in zip(run(window, sinks), want)), (window, sinks)
    some = run(100, lk)
    for sinks in (2 ** 31, MOST - 200, MOST):
        assert all(torch.equal(x, y) for x, y in zip(run(100, sinks), some)), sinks


def test_more_rows_of_logits_than_a_launch_counts():
    """Above 2^32 threads, 2^24 workgroups of 256, a launch leaves workgroups out without an error: the rows go in two."""
    rows = 2 ** 24 + 5
    z = torch.tensor([[0x40, 0x30, 0x40]], dtype=torch.uint8, device="cuda")
    targets = torch.tensor([1], dtype=torch.int32, device="cuda")
    g = torch.ones(1, device="cuda")
    one = pn.posit_token_logprob_fwd(z, targets, "p8", top=1)
    many = pn.posit_token_logprob_fwd(z.repeat(rows, 1), targets.repeat(rows), "p8", top=1)
    for a, b in zip(one, many):
        assert (b == a).all()
    want = pn.posit_token_logprob_bwd(z, targets, one[1], one[2], g, g, "p8", "bf16")
    got = pn.posit_token_logprob_bwd(z.repeat(rows, 1), targets.repeat(rows), many[1], many[2], g.repeat(rows), g.repeat(rows), "p8", "bf16")
    assert (got == want).all()
