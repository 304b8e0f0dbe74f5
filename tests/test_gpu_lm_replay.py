"""Caches cut into as many parts as the join takes, and the operators recorded into a HIP graph: every replay against the eager result."""
import numpy as np
import pytest
import torch

import paper_2105_00053_amd as pn
from lm_util import normal, to_format
from test_gpu_lm_attention import _compare, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens", [[60001], [33000], [17], [0]])
def test_a_single_sequence_in_many_parts(lens):
    _, q, k, v, do = _inputs(1, 1, 60001, 2, 1, 16, "bf16", "p8_1", 31)
    _compare(q, k, v, do, "bf16", "p8_1", "f32", lens=lens, back=False)


def test_graph_replays():
    rng = np.random.default_rng(32)
    b, l, h, hk, d, vocab = 2, 70, 4, 2, 32, 40000
    x = to_format(normal(rng, (b * l, h * d)), "p8_2")
    res = to_format(normal(rng, (b * l, h * d)), "p16")
    w = to_format(1 + 0.1 * normal(rng, (h * d,)), "p16")
    k, v = (to_format(normal(rng, (b, l, hk, d)), "p8_2") for _ in range(2))
    long_k, long_v = (to_format(normal(rng, (b, 3000, hk, d)), "p8_2") for _ in range(2))
    z = to_format(normal(rng, (b, vocab)), "p16")
    targets = torch.tensor([5, vocab - 1], dtype=torch.int32, device="cuda")
    g = torch.ones(b, dtype=torch.float32, device="cuda")

    def step():
        y, scale, stream, rstd = pn.posit_rmsnorm_fwd(x, w, "p8_2", "p16", "p8_2", res=res, fres="p16", scaled=True)
        q = y.view(b, l, h, d)
        o, lse, _ = pn.posit_attention_fwd(q, k, v, "p8_2", "p8_2", "p8_2", window=20, sinks=2)
        dq, dk, dv = pn.posit_attention_bwd(o, q, k, v, o, lse, "p8_2", "p8_2", "p8_2", "p8_2", "bf16", window=20, sinks=2)
        dx, dw = pn.posit_rmsnorm_bwd(dq.view(b * l, h * d), stream, w, rstd, "bf16", "p16", "p16", "bf16", "f32")
        token, _, _ = pn.posit_attention_fwd(q[:, :1], long_k, long_v, "p8_2", "p8_2", "f32")
        lp, z_lse, ent, top, index = pn.posit_token_logprob_fwd(z, targets, "p16", top=7)
        dz = pn.posit_token_logprob_bwd(z, targets, z_lse, ent, g, g, "p16", "f32")
        return [pn.posit_scale_rows(y, scale, "p8_2", "f32"), o, lse, dk, dv, dx, dw, token, lp, z_lse, ent, top, index, dz]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(4):
        r = np.random.default_rng(seed)
        x.copy_(to_format(normal(r, (b * l, h * d)), "p8_2"))
        z.view(torch.int16).copy_(to_format(normal(r, (b, vocab)), "p16").view(torch.int16))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = step()
        torch.cuda.synchronize()
        for n, (a, c) in enumerate(zip(got, want)):
            a, c = (t.view(torch.int16) if t.dtype == torch.uint16 else t for t in (a, c))
            assert torch.equal(a, c), (seed, n)


@pytest.mark.parametrize("b,l,hq,hkv,d", [(1, 331, 5, 1, 40), (2, 520, 2, 1, 64), (1, 300, 8, 1, 128), (1, 700, 6, 2, 96)])
def test_gradients_of_few_heads_over_many_rows(b, l, hq, hkv, d):
    """Tiles of keys whose rows are shared out over workgroups."""
    _, q, k, v, do = _inputs(b, l, l, hq, hkv, d, "p8_2", "p8_2", 33)
    _compare(q, k, v, do, "p8_2", "p8_2", "bf16")
    _compare(q, k, v, do, "p8_2", "p8_2", "f32", window=53, sinks=4, lens=[l - 97 * (i + 1) for i in range(b)])


def test_nar_in_a_row_of_a_shared_tile():
    """A NaR in one row of the output's gradient: dV of the keys that the row sees is NaN, of the others what it is without."""
    l, d = 400, 32
    _, q, k, v, do = _inputs(1, l, l, 4, 1, d, "p8_2", "p8_2", 34)
    o, lse, copy = pn.posit_attention_fwd(q, k, v, "p8_2", "p8_2", "bf16", fcopy="f32", window=60)
    back = lambda g: pn.posit_attention_bwd(g, q, k, v, copy, lse, "p8_2", "p8_2", "p8_2", "f32", "f32", window=60)  # noqa: E731
    clean = back(do)
    bad = do.clone()
    bad[0, 200, 1, 7] = 128
    got = back(bad)
    sees = torch.zeros(l, dtype=torch.bool, device="cuda")
    sees[141:201] = True
    assert torch.isnan(got[2][0, sees, 0, 7]).all()
    assert torch.equal(got[2][0, ~sees], clean[2][0, ~sees]) and torch.equal(got[1][0, ~sees], clean[1][0, ~sees])
    assert torch.isnan(got[1][0, sees]).all()
