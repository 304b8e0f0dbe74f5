"""Weights' gradients where queries, keys or both have no heads: sums over nothing."""
import ctypes

import numpy as np
import pytest
import torch

import lm_util as lu
import paper_2105_00053_amd as pn
from paper_2105_00053_amd import binding, generate

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("hq,hkv", [(0, 2), (3, 0), (0, 0)])
def test_gradients_of_weights_without_heads_are_zeros(monkeypatch, native, hq, hkv):
    generate._load()
    if native and binding._native is None:
        pytest.skip("the extension module is not built")
    if not native:
        monkeypatch.setattr(binding, "_native", None)
    rng = np.random.default_rng(hq + hkv)
    t, d = 5, 32
    x, g = (lu.to_format(lu.normal(rng, (t, hq + hkv + 1, d)), "bf16")[:, :hq + hkv] for _ in range(2))
    q, k = x[:, :hq], x[:, hq:]
    w = [lu.to_format(1 + lu.normal(rng, (d,), 0.2), "f32") for _ in range(2)]
    how = dict(wq=w[0], wk=w[1], fw="f32")
    _, _, rstd = pn.posit_qk_norm_rope_fwd(q, k, "bf16", "f32", **how)
    for _ in range(3):  # memory that held something else
        junk = [torch.full((d,), 7.0, device="cuda") for _ in range(8)]
        del junk
        dq, dk, dwq, dwk = pn.posit_qk_norm_rope_bwd(g[:, :hq], g[:, hq:], q, k, rstd, "bf16", "bf16", "f32", **how)
        assert dq.shape == q.shape and dk.shape == k.shape and dwq.shape == dwk.shape == (d,)
        assert bool(dwq.any()) == (hq > 0) and bool(dwk.any()) == (hkv > 0)
    if hq + hkv:  # the same of the heads that there are, alone
        alone = pn.posit_qk_norm_rope_bwd(g, None, x, None, rstd, "bf16", "bf16", "f32", wq=w[0] if hq else w[1], fw="f32")
        assert torch.equal(alone[2], dwq if hq else dwk) and torch.equal(alone[0], dq if hq else dk)


@pytest.mark.parametrize("hq,hkv", [(0, 2), (3, 0)])
def test_the_c_call_writes_both(hq, hkv):
    rng = np.random.default_rng(3)
    t, d, h = 4, 16, hq + hkv
    x, g = (lu.to_format(lu.normal(rng, (t, h, d)), "f32") for _ in range(2))
    w = lu.to_format(1 + lu.normal(rng, (d,), 0.2), "f32")
    _, _, rstd = pn.posit_qk_norm_rope_fwd(x, None, "f32", "f32", wq=w, fw="f32")
    desc = generate.HeadsDesc(t, hq, hkv, d, 0, h * d, d, h * d, d, h * d, d, h * d, d, 0, 0.0)
    L = generate._load()
    n = L.posit_qk_norm_rope_bwd_workspace(ctypes.byref(desc))
    work, dx, dwq, dwk = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty_like(x), torch.full((d,), 7.0, device="cuda"), torch.full((d,), 7.0, device="cuda")
    p = lambda a, some=True: a.data_ptr() if some else None  # noqa: E731
    status = L.posit_qk_norm_rope_bwd(generate._stream(), 100, 100, 100, 100, 100, ctypes.byref(desc), p(g, hq), p(g, hkv), p(x, hq), p(x, hkv), p(w, hq), p(w, hkv), p(rstd), None, None,
                                      p(dx, hq), p(dx, hkv), p(dwq), p(dwk), p(work), n)
    torch.cuda.synchronize()
    assert status == 0 and bool(dwq.any()) == (hq > 0) and bool(dwk.any()) == (hkv > 0)
