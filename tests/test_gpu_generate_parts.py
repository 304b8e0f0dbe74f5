"""Rows of logits taken whole and in parts give the same: a row among many, which are whole, and alone or among few, where long rows go in parts."""
import numpy as np
import pytest
import torch

import generate_util as gu
import lm_util as lu
import paper_2105_00053_amd as pn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,vocab,rows", [("p8", 140001, 40), ("p8_2", 131081, 20), ("p16", 20011, 30), ("p12_2", 66003, 70), ("f32", 33001, 40), ("bf16", 70001, 80)])
def test_a_row_among_many_is_the_row_alone(fmt, vocab, rows):
    rng = np.random.default_rng(vocab)
    z, u = lu.to_format(lu.normal(rng, (rows, vocab), 2.5), fmt), gu.dev(rng.random(rows), np.float32)
    how = dict(temperature=gu.dev(0.5 + rng.random(rows), np.float32), top_k=gu.dev(rng.integers(0, 200, rows), np.int32), top_p=gu.dev(0.8 + 0.2 * rng.random(rows), np.float32),
               min_p=gu.dev(0.02 * rng.random(rows), np.float32))
    many = pn.posit_sample(z, u, fmt, **how)
    for first, last in ((0, 1), (3, 5)):
        few = pn.posit_sample(z[first:last], u[first:last], fmt, **{name: t[first:last] for name, t in how.items()})
        assert all(torch.equal(a[first:last], b) for a, b in zip(many, few))
