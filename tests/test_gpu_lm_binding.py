"""The binding's two ways to the library, in C++ and in Python, give the same tensors."""
import pytest
import torch

import paper_2105_00053_amd as pn
from paper_2105_00053_amd import binding

pytestmark = pytest.mark.gpu


def _calls():
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, res, w = pn.posit_round(rand(5, 70), "p8_1"), pn.posit_round(rand(5, 70), "p16"), pn.posit_round(rand(70), "p16")
    dy = rand(5, 70).to(torch.bfloat16)
    q, k, v = (pn.posit_round(rand(2, 9, h, 40), "p8_1") for h in (4, 2, 2))
    do = pn.posit_round(rand(2, 9, 4, 40), "p8_1")
    lens = torch.tensor([9, 5], dtype=torch.int32, device="cuda")
    z = pn.posit_round(rand(4, 300), "p16")
    y = torch.tensor([3, -1, 299, 0], dtype=torch.int32, device="cuda")
    g1, g2 = rand(4), rand(4)

    def run():
        out = []
        for scaled in (False, True):
            n = pn.posit_rmsnorm_fwd(x, w, "p8_1", "p16", "p8_2", res=res, fres="p16", scaled=scaled)
            out += list(n)
        out += list(pn.posit_rmsnorm_fwd(x[:, 3:], w[3:].clone(), "p8_1", "p16", "bf16"))
        out.append(pn.posit_scale_rows(n[0], n[1], "p8_2", "bf16"))
        out += list(pn.posit_rmsnorm_bwd(dy, n[2], w, n[3], "bf16", "p16", "p16", "bf16", "f32", dres=dy))
        out += list(pn.posit_rmsnorm_bwd(dy, n[2], w, n[3], "bf16", "p16", "p16", "p16", "f32", want_dw=False))
        o = pn.posit_attention_fwd(q, k, v, "p8_1", "p8_1", "bf16", window=4, sinks=1, lens=lens, fcopy="f32")
        out += list(o) + list(pn.posit_attention_fwd(q[:, :1], k, v, "p8_1", "p8_1", "p8_1"))
        out += list(pn.posit_attention_bwd(do, q, k, v, o[2], o[1], "p8_1", "p8_1", "p8_1", "f32", "bf16", window=4, sinks=1, lens=lens))
        lp = pn.posit_token_logprob_fwd(z, y, "p16", inv_temperature=0.5, top=3)
        out += list(lp) + list(pn.posit_token_logprob_fwd(z, None, "p16"))
        out.append(pn.posit_token_logprob_bwd(z, y, lp[1], lp[2], g1, g2, "p16", "p8_2", inv_temperature=0.5))
        return out

    return run


def test_both_ways_agree(monkeypatch):
    run = _calls()
    a = run()
    if binding._native is None:
        pytest.skip("the extension module is not built")
    monkeypatch.setattr(binding, "_native", None)
    b = run()
    assert len(a) == len(b)
    for s, t in zip(a, b):
        assert (s is None) == (t is None)
        if s is not None:
            assert s.dtype == t.dtype and s.shape == t.shape and s.device == t.device and torch.equal(s.cpu().view(torch.uint8), t.cpu().view(torch.uint8))


def test_refusals_are_errors_both_ways(monkeypatch):
    x = torch.zeros((4, 8), dtype=torch.uint8, device="cuda")
    w = torch.ones(8, device="cuda")
    z = torch.zeros((4, 8), device="cuda")

    def refused():
        for call in (lambda: pn.posit_rmsnorm_fwd(x, w, "p8", "f32", "p32"), lambda: pn.posit_rmsnorm_fwd(x, w[:7], "p8", "f32", "p8"),
                     lambda: pn.posit_rmsnorm_fwd(x, w, "p8", "f32", "p8", eps=-1.0), lambda: pn.posit_rmsnorm_fwd(x.t(), w[:4], "p8", "f32", "p8"),
                     lambda: pn.posit_scale_rows(x, w, "p8", "f32"), lambda: pn.posit_token_logprob_fwd(z, None, "f32", top=65),
                     lambda: pn.posit_token_logprob_fwd(z, None, "f32", inv_temperature=0.0),
                     lambda: pn.posit_attention_fwd(x.reshape(1, 4, 2, 4), x.reshape(1, 4, 2, 4), x.reshape(1, 2, 4, 4), "p8", "p8", "bf16"),
                     lambda: pn.posit_attention_fwd(x.reshape(1, 4, 2, 4), x.reshape(1, 4, 2, 4), x.reshape(1, 4, 2, 4), "p8", "p8", "bf16", window=-1),
                     lambda: pn.posit_attention_fwd(z.reshape(1, 4, 2, 4), z.reshape(1, 4, 2, 4), z.reshape(1, 4, 2, 4), "f32", "f32", "bf16")):
            with pytest.raises(pn.PositError):
                call()

    refused()
    monkeypatch.setattr(binding, "_native", None)
    refused()
