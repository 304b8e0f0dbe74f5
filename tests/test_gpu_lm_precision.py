"""What the operators promise beyond the plain bounds: 16 bits of each probability where an output keeps more than bfloat16 and for few queries, long windows
and prompts on filled caches, wide rows."""
import numpy as np
import pytest
import torch

import paper_2105_00053_amd as pn
from lm_util import U, attention, check, norm_bwd, norm_fwd, normal, to_format, values
from test_gpu_lm_attention import _inputs

pytestmark = pytest.mark.gpu


def _forward(q, k, v, fq, fkv, fout, fcopy, window, sinks, lens):
    d = q.shape[3]
    lt = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse, copy = pn.posit_attention_fwd(q, k, v, fq, fkv, fout, window=window, sinks=sinks, lens=lt, fcopy=fcopy)
    w = attention(values(q, fq), values(k, fkv), values(v, fkv), np.float64(np.float32(1 / np.sqrt(d))), window, sinks, lens, 16)
    check(lse, w["lse"], w["s_lse"], "f32", "lse")
    check(o, w["o"], w["s_o"], fout, "o")
    if copy is not None:
        check(copy, w["o"], w["s_o"], fcopy, "o_copy")


@pytest.mark.parametrize("d", [40, 64, 128])
@pytest.mark.parametrize("fkv", ["p8_1", "p12_2", "bf16"])
def test_sixteen_bits_of_a_probability(d, fkv):
    """A copy in binary32 beside bfloat16 outputs of many queries, and every output of few."""
    for lq, fout, fcopy in ((90, "bf16", "f32"), (90, "bf16", "p16"), (1, "bf16", None), (1, "bf16", "f32"), (7, "f32", None), (1, "p16", "bf16")):
        _, q, k, v, _ = _inputs(2, lq, 200, 4, 2, d, "bf16", fkv, 71)
        _forward(q, k, v, "bf16", fkv, fout, fcopy, 60, 3, [200, 133])


@pytest.mark.parametrize("lq,lk,window,sinks", [(1, 6000, 3000, 50), (3, 6000, 4096, 4), (40, 4000, 3000, 50), (150, 2500, 900, 70), (150, 1400, 0, 0), (20, 3000, 2999, 1)])
def test_long_windows_and_prompts_on_filled_caches(lq, lk, window, sinks):
    _, q, k, v, _ = _inputs(2, lq, lk, 2, 1, 64, "p8_1", "p8_1", 72)
    _forward(q, k, v, "p8_1", "p8_1", "f32", None, window, sinks, [lk, lk - 777])


@pytest.mark.parametrize("rows,cols", [(700, 8200), (300, 12288)])
def test_gradients_of_many_wide_rows(rows, cols):
    rng = np.random.default_rng([73, rows])
    h, w = to_format(normal(rng, (rows, cols)), "p16"), to_format(1 + normal(rng, cols, 0.1), "p16")
    dy, dres = to_format(normal(rng, (rows, cols)), "bf16"), to_format(normal(rng, (rows, cols)), "bf16")
    y, _, _, rstd = pn.posit_rmsnorm_fwd(h, w, "p16", "p16", "bf16")
    hv, r, t = norm_fwd(values(h, "p16"), None, values(w, "p16"), 1e-6, None)
    k = (cols / 64 + 32) * U
    check(rstd, r, k * r, "f32", "rstd")
    check(y, t * r[:, None], k * np.abs(t * r[:, None]), "bf16", "y")
    dx, dw = pn.posit_rmsnorm_bwd(dy, h, w, rstd, "bf16", "p16", "p16", "bf16", "f32", dres=dres, fdres="bf16")
    wx, ww, sx, sw = norm_bwd(values(dy, "bf16"), hv, values(w, "p16"), values(rstd, "f32"), values(dres, "bf16"))
    check(dx, wx, sx, "bf16", "dx")
    check(dw, ww, sw, "f32", "dw")
