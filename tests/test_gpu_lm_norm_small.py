"""Scaled RMS norm of rows whose largest magnitude is near the end of binary32's range."""
import numpy as np
import pytest
import torch

import paper_2105_00053_amd as pn
from lm_util import U, check, normal, to_format, values

pytestmark = pytest.mark.gpu

EXPONENTS = [-149, -148, -140, -128, -127, -126, -125, -124, -123, -100, 0, 100, 120]


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [5, 700, 8300])
@pytest.mark.parametrize("fy", ["p8", "p8_2", "p16"])
def test_rows_of_any_magnitude(fmt, cols, fy):
    """The largest |t| is 1.5 * 2^e (2^e where that is the smallest number), the others lie below by up to 2^6: patterns are the rounding of t * 2^(2-e), the scale is
    rstd * 2^(e-2), where a subnormal result has its own rounding.  Weights of one, so that t is h exactly."""
    rng = np.random.default_rng([51, cols])
    exps = [e for e in EXPONENTS if fmt == "f32" or e >= -133]  # bfloat16 has numbers from 2^-133
    x = np.zeros((len(exps), cols), np.float32)
    for r, e in enumerate(exps):
        x[r] = np.ldexp(rng.uniform(-1, 1, cols) * np.exp2(-rng.integers(0, 7, cols)), e).astype(np.float32)
        x[r, cols // 2] = np.ldexp(1.0 if e == -149 or (fmt == "bf16" and e == -133) else -1.5, e)
    xt = to_format(x, fmt)
    y, scale, _, rstd = pn.posit_rmsnorm_fwd(xt, torch.ones(cols, device="cuda"), fmt, "f32", fy, eps=0.25, scaled=True)
    t = values(xt, fmt)
    top = np.floor(np.log2(np.abs(t).max(axis=1)))
    up = np.exp2(2 - top)[:, None]
    check(y, t * up, 0.0, fy, "patterns")
    small = np.array([e < 60 for e in exps])  # the squares of the others do not fit binary32
    r = 1.0 / np.sqrt((t * t).mean(axis=1) + 0.25)
    k = (cols / 64 + 32) * U
    check(rstd[torch.from_numpy(small).cuda()], r[small], (k * r)[small], "f32", "rstd")
    want = values(rstd, "f32") * np.exp2(top - 2)
    check(scale, want, 0.0, "f32", "scale")
