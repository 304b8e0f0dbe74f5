"""Zero-sized problems: results that would stay unwritten are refused or filled in, both ways through the binding."""
import pytest
import torch

import paper_2105_00053_amd as pn
from paper_2105_00053_amd import binding

pytestmark = pytest.mark.gpu


def _calls():
    q, k = torch.zeros((2, 3, 4, 0), dtype=torch.uint8, device="cuda"), torch.zeros((2, 5, 2, 0), dtype=torch.uint8, device="cuda")
    x, w = torch.zeros((3, 0), dtype=torch.uint8, device="cuda"), torch.ones(0, device="cuda")
    for call in (lambda: pn.posit_attention_fwd(q, k, k, "p8", "p8", "bf16"), lambda: pn.posit_rmsnorm_fwd(x, w, "p8", "f32", "p8"),
                 lambda: pn.posit_rmsnorm_fwd(x, w, "p8", "f32", "p8", scaled=True), lambda: pn.posit_token_logprob_fwd(x, None, "p8")):
        with pytest.raises(pn.PositError):
            call()
    o, lse, copy = pn.posit_attention_fwd(q[:, :0], k, k, "p8", "p8", "bf16", fcopy="f32")
    assert o.shape == copy.shape == (2, 0, 4, 0) and lse.shape == (2, 4, 0)
    y, scale, _, rstd = pn.posit_rmsnorm_fwd(x[:0], w, "p8", "f32", "p8", scaled=True)
    assert y.shape == (0, 0) and scale.shape == rstd.shape == (0,)
    dx, dw = pn.posit_rmsnorm_bwd(x[:0].expand(0, 0), x[:0], w, rstd, "p8", "p8", "f32", "p8", "f32")
    assert dx.shape == (0, 0) and dw.shape == (0,)
    ones = torch.ones(7, device="cuda")
    z = torch.zeros((0, 7), dtype=torch.uint8, device="cuda")
    dx, dw = pn.posit_rmsnorm_bwd(z, z, ones, torch.ones(0, device="cuda"), "p8", "p8", "f32", "p8", "p16")
    assert dx.shape == (0, 7) and (dw.cpu().view(torch.int16) == 0).all()


def test_both_ways(monkeypatch):
    _calls()
    monkeypatch.setattr(binding, "_native", None)
    _calls()
