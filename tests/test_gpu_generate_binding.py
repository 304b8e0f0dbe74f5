"""The binding's two ways to the library, in C++ and in Python, give the same tensors and refuse alike; the calls recorded into a HIP graph, every replay against the eager result;
calls on a stream of their own."""
import numpy as np
import pytest
import torch

import generate_util as gu
import lm_util as lu
import paper_2105_00053_amd as pn
from paper_2105_00053_amd import binding

pytestmark = pytest.mark.gpu


class Step:
    """A step of two sequences from the rows of a product to tokens, and the heads' backward pass; all inputs are tensors that stay."""

    def __init__(self, seed=1, long=40):
        rng = np.random.default_rng(seed)
        self.rng, self.lens = rng, [long, 9]
        self.table, pages = gu.tables(rng, self.lens, 16)
        self.table = gu.dev(self.table)
        self.x = lu.to_format(lu.normal(rng, (3, 8, 32)), "p8_1")
        self.w = [lu.to_format(1 + lu.normal(rng, (32,), 0.1), "p16") for _ in range(2)]
        self.freq, self.pos = pn.rope_frequencies(24), torch.tensor([5, -1, 70000], dtype=torch.int32, device="cuda")
        self.g = lu.to_format(lu.normal(rng, (3, 6, 32)), "bf16")
        self.lens, self.starts = gu.dev(self.lens, np.int32), gu.dev([0, 2, 3], np.int32)
        self.pages = {f: pn.posit_cache_pages(pages, 2, 16, 32, f) for f in gu.CACHES}
        self.z, self.u = lu.to_format(lu.normal(rng, (3, 20000), 2.0), "p16"), gu.dev(rng.random(3), np.float32)
        self.limits = dict(temperature=gu.dev([0.7, 1, 0], np.float32), top_k=gu.dev([0, 50, 3], np.int32), top_p=gu.dev([0.9, 1, 0.5], np.float32), min_p=gu.dev([0, 0.01, 0], np.float32))

    def run(self):
        x, out = self.x, []
        q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
        how = dict(positions=self.pos, inv_freq=self.freq, wq=self.w[0], wk=self.w[1], fw="p16")
        yq, yk, rstd = pn.posit_qk_norm_rope_fwd(q, k, "p8_1", "bf16", **how)
        out += [yq, yk, rstd, *pn.posit_qk_norm_rope_fwd(q, None, "p8_1", "p8_2", positions=self.pos, inv_freq=self.freq, neighbours=True)]
        out += pn.posit_qk_norm_rope_bwd(self.g[:, :4], self.g[:, 4:], q, k, rstd, "bf16", "p8_1", "p8_2", **how)
        out += pn.posit_qk_norm_rope_bwd(self.g[:, :4], self.g[:, 4:], q, k, rstd, "bf16", "p8_1", "f32", want_dw=False, **how)
        for f, pages in self.pages.items():
            r = pn.posit_cache_append(k, v, *pages, self.table, self.lens, "p8_1", f, starts=self.starts, q=q, fq="bf16", inv_freq=self.freq, wq=self.w[0], wk=self.w[1], fw="p16")
            out += [r, pages[0].clone(), pages[1].clone(), *pn.posit_cache_read(*pages, self.table, self.lens, 41, 32, f, "bf16")]
            out += pn.posit_attention_paged(r, *pages, self.table, self.lens, "bf16", f, "p8_1", starts=self.starts, most=2, window=20, sinks=1)
            out += pn.posit_attention_paged(r[:2], *pages, self.table, self.lens, "bf16", f, "f32", longest=33, scale=0.2)
        out.append(pn.posit_cache_append(k[:2], v[:2], *self.pages["p8"], self.table, self.lens, "p8_1", "p8"))
        out += pn.posit_sample(self.z, self.u, "p16", **self.limits) + pn.posit_sample(self.z[:, :3000], self.u, "p16")
        return out


def bits(t):
    return t.cpu().contiguous().view(torch.uint8)


def same(a, b):
    assert len(a) == len(b)
    for n, (s, t) in enumerate(zip(a, b)):
        assert (s is None) == (t is None), n
        if s is not None:
            assert s.dtype == t.dtype and s.shape == t.shape and torch.equal(bits(s), bits(t)), n


def test_both_ways_agree(monkeypatch):
    step = Step()
    a = step.run()
    if binding._native is None:
        pytest.skip("the extension module is not built")
    monkeypatch.setattr(binding, "_native", None)
    same(a, step.run())


def test_refusals_are_errors_both_ways(monkeypatch):
    s = Step()
    q, k, v = s.x[:, :4], s.x[:, 4:6], s.x[:, 6:]
    kc, vc = s.pages["p8"]
    ints, real = s.pos, s.u

    def refused():
        for call in (lambda: pn.posit_qk_norm_rope_fwd(q, k, "p8_1", "p32"), lambda: pn.posit_qk_norm_rope_fwd(q, k[:2], "p8_1", "bf16"),
                     lambda: pn.posit_qk_norm_rope_fwd(q, k, "p8_1", "bf16", wq=s.w[0], fw="p16"), lambda: pn.posit_qk_norm_rope_fwd(q, k, "p8_1", "bf16", positions=ints),
                     lambda: pn.posit_qk_norm_rope_fwd(q, k, "p8_1", "bf16", positions=ints[:2], inv_freq=s.freq),
                     lambda: pn.posit_qk_norm_rope_fwd(q, k, "p8_1", "bf16", positions=ints, inv_freq=s.freq.float()),
                     lambda: pn.posit_qk_norm_rope_fwd(q, k, "p8_1", "bf16", wq=s.w[0], wk=s.w[1], fw="p16", eps=-1.0),
                     lambda: pn.posit_qk_norm_rope_bwd(q, k[:2], q, k, None, "p8_1", "p8_1", "bf16"),
                     lambda: pn.posit_qk_norm_rope_bwd(q, k, q, k, None, "p8_1", "p8_1", "bf16", wq=s.w[0], wk=s.w[1], fw="p16"),
                     lambda: pn.posit_cache_append(k, v, kc, vc, s.table, s.lens, "p8_1", "p8"),                                   # three rows, two sequences
                     lambda: pn.posit_cache_append(k, v, kc, vc[:1], s.table, s.lens, "p8_1", "p8", starts=s.starts),
                     lambda: pn.posit_cache_append(k, v, kc, vc, s.table, s.lens[:1], "p8_1", "p8", starts=s.starts),
                     lambda: pn.posit_cache_append(k, v, kc, vc, s.table, s.lens, "p8_1", "p16", starts=s.starts),
                     lambda: pn.posit_cache_append(k, v, kc, vc, s.table, s.lens, "p8_1", "p8", starts=s.starts, wk=s.w[0], fw="p16", q=q),
                     lambda: pn.posit_cache_append(k, v[:, :, :16], kc, vc, s.table, s.lens, "p8_1", "p8", starts=s.starts),
                     lambda: pn.posit_cache_append(k, v, kc, vc, s.table.long(), s.lens, "p8_1", "p8", starts=s.starts),
                     lambda: pn.posit_cache_read(kc, vc, s.table, s.lens, -1, 32, "p8", "f32"), lambda: pn.posit_cache_read(kc, vc, s.table, s.lens, 9, 40, "p8", "f32"),
                     lambda: pn.posit_cache_read(kc, vc, s.table, None, 9, 32, "p8", "f32"),
                     lambda: pn.posit_attention_paged(q, kc, vc, s.table, s.lens, "p8_1", "p8", "f32"), lambda: pn.posit_attention_paged(q[:2, :3], kc, vc, s.table, s.lens, "p8_1", "p8", "f32"),
                     lambda: pn.posit_attention_paged(q[:2], kc, vc, s.table, s.lens, "p8_1", "p8", "f32", most=2000),
                     lambda: pn.posit_attention_paged(q[:2], kc, vc, s.table, s.lens, "p8_1", "p8", "f32", window=-1),
                     lambda: pn.posit_attention_paged(q[:2].float(), kc, vc, s.table, s.lens, "f32", "p8", "f32"),
                     lambda: pn.posit_sample(s.z, real[:2], "p16"), lambda: pn.posit_sample(s.z, real, "p16", top_k=real), lambda: pn.posit_sample(s.z, None, "p16"),
                     lambda: pn.posit_sample(s.z.view(torch.uint8), real, "p16"), lambda: pn.posit_sample(s.z, real, "p16", workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))):
            with pytest.raises(pn.PositError):
                call()

    refused()
    monkeypatch.setattr(binding, "_native", None)
    refused()


def test_graph_replays():
    step = Step(2, long=3000)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step.run()
    for seed in range(4):
        r = np.random.default_rng(seed)
        step.x.copy_(lu.to_format(lu.normal(r, (3, 8, 32)), "p8_1"))
        step.z.view(torch.int16).copy_(lu.to_format(lu.normal(r, (3, 20000), 2.0), "p16").view(torch.int16))
        step.u.copy_(gu.dev(r.random(3), np.float32))
        step.lens.copy_(gu.dev([2500 + 100 * seed, 9 - seed], np.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = [None if t is None else t.clone() for t in out]
        same(got, step.run())
        torch.cuda.synchronize()


def test_two_streams_at_once():
    """Two steps, each on its own tensors and stream, as they are one after the other."""
    steps = [Step(3, long=2000), Step(4, long=1500)]
    want = [s.run() for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    got = []
    for s, stream in zip(steps, streams):
        with torch.cuda.stream(stream):
            got.append([s.run() for _ in range(3)])
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for one in g:
            same(w, one)
