"""Log probabilities at temperatures near zero, and rows with a pitch bit for bit."""
import numpy as np
import pytest
import torch

import paper_2105_00053_amd as pn
from lm_util import U, check, logprob, normal, to_format, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["p8", "p8_2", "p10_1", "p10_2", "p12_1", "p12_2", "p16", "bf16", "f32"])
@pytest.mark.parametrize("vocab", [7, 900, 40000])
def test_zeros_are_zeros_at_any_temperature(fmt, vocab):
    """Rows whose largest logits are zeros (in one row the only ones that are not negative, in one all, in one behind a single larger one): a zero times any
    inverse temperature is zero."""
    rng = np.random.default_rng([61, vocab])
    z = np.zeros((3, vocab), np.float32)
    z[0] = np.where(rng.random(vocab) < 0.5, 0.0, -1.0 - np.abs(normal(rng, vocab)))
    z[0, 0], z[0, vocab - 1] = 0.0, -2.0
    z[2, vocab // 2] = 1.0
    zt = to_format(z, fmt)
    y = torch.tensor([0, vocab - 1, vocab // 2], dtype=torch.int32, device="cuda")
    for tau in (1e-3, 1.0, 1e10, 1e19, 1e30):
        lp, lse, ent, tlp, tix = pn.posit_token_logprob_fwd(zt, y, fmt, inv_temperature=tau, top=3)
        want = logprob(values(zt, fmt), y.cpu().numpy(), np.float64(np.float32(tau)), 3)
        check(lse, want["lse"], want["slack"], "f32", "lse")
        check(lp, want["logprob"], want["slack"] + 4 * U * np.abs(want["logprob"]), "f32", "logprob")
        check(ent, want["entropy"], want["s_entropy"], "f32", "entropy")
        assert np.array_equal(tix.cpu().numpy(), want["top_index"])


@pytest.mark.parametrize("fmt,cols", [("p16", 5003), ("p8_2", 911), ("f32", 40001), ("bf16", 33001), ("p12_2", 70003), ("p8", 66001)])
def test_rows_with_a_pitch_bit_for_bit(fmt, cols):
    """How a row is cut depends on its format and length alone, not on its address: views give what their copies give."""
    rng = np.random.default_rng(62)
    big = to_format(normal(rng, (6, cols + 9), 2), fmt)
    z = big[1:5, 3:3 + cols]
    y = torch.from_numpy(rng.integers(0, cols, 4).astype(np.int32)).cuda()
    g, h = (torch.from_numpy(normal(rng, 4)).cuda() for _ in range(2))
    a = pn.posit_token_logprob_fwd(z, y, fmt, top=5)
    b = pn.posit_token_logprob_fwd(z.contiguous(), y, fmt, top=5)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    for fg in ("bf16", "f32"):
        assert torch.equal(pn.posit_token_logprob_bwd(z, y, a[1], a[2], g, h, fmt, fg), pn.posit_token_logprob_bwd(z.contiguous(), y, a[1], a[2], g, h, fmt, fg))
