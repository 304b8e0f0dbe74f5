"""A cache of no pages: every token of a sequence lies in a page that is none, as for posit_cache_read."""
import numpy as np
import pytest
import torch

import generate_util as gu
import lm_util as lu
import paper_2105_00053_amd as pn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fc", ["p8_1", "bf16", "f4"])
@pytest.mark.parametrize("columns,fout", [(4, "f32"), (400, "p8_2")])
def test_rows_that_see_a_token_are_nan(fc, columns, fout):
    rng = np.random.default_rng(columns)
    hq, hkv, d, page = 6, 2, 40, 16
    k, v = pn.posit_cache_pages(0, hkv, page, d, fc)
    assert k.shape[0] == 0
    lens, new = [columns * page, 0, 2, 30, -4], [1, 1, 3, 2, 1]
    q = lu.to_format(lu.normal(rng, (sum(new), hq, d)), "bf16")
    starts = np.concatenate([[0], np.cumsum(new)])
    table = gu.dev(rng.integers(-1, 3, (len(lens), columns)), np.int32)
    args = (table, gu.dev(lens, np.int32))
    for how in (dict(), dict(window=5, sinks=2)):
        o, lse = pn.posit_attention_paged(q, k, v, *args, "bf16", fc, fout, starts=gu.dev(starts, np.int32), most=3, **how)
        o = lu.values(o, fout)
        for b, n in enumerate(new):
            for i in range(n):
                row, sees = starts[b] + i, max(lens[b], 0) - n + i >= 0
                assert np.isnan(o[row]).all() if sees else not o[row].any(), (b, i)
                assert torch.isnan(lse[row]).all() if sees else torch.isneginf(lse[row]).all(), (b, i)
    dense, _ = pn.posit_cache_read(k, v, *args, 8, d, fc, "f32")
    assert torch.isnan(dense[0]).all() and not dense[1].any() and torch.isnan(dense[2, :2]).all() and not dense[2, 2:].any()
    # single rows, in order
    o, lse = pn.posit_attention_paged(q[:5], k, v, *args, "bf16", fc, "f32")
    assert torch.isnan(o[[0, 2, 3]]).all() and not o[[1, 4]].any() and torch.isneginf(lse[[1, 4]]).all()
