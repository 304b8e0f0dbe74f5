"""What the token model's step hands from one operator to the next keeps the operators' own accuracy."""
import numpy as np
import pytest

import lm_util as lu
from paper_2105_00053_amd import lm, lm_step
from test_gpu_lm_step import make, tokens_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("how", [{}, {"window": 9, "sinks": 2}, {"compute": "p8_1"}, {"compute": "p12_2", "window": 5}])
def test_attention_gradients_are_those_of_the_unrounded_output(monkeypatch, how):
    """dq, dk and dv of the step against the formula in 64 bits on the q, k, v and dO that it computed: every one within its own rounding and the kernels'
    bound.  A row's sum of dO * o taken from the o of 8 bits would move all scores' gradients of that row by up to 1/16 of it."""
    calls = []

    def watched(*args, **kw):
        calls.append((args, lm_bwd(*args, **kw)))
        return calls[-1][1]

    lm_bwd = lm.posit_attention_bwd
    monkeypatch.setattr(lm, "posit_attention_bwd", watched)
    net, g = make(11, **how)
    tokens, targets = tokens_of(g, 2, 41)
    lm_step.gradients(net, tokens, targets)
    (args, grads), = calls
    do, q, k, v = (lu.values(lm_step._movable(t), net.compute) for t in args[:4])
    w = lu.attention(q, k, v, np.float64(np.float32(1 / np.sqrt(net.d))), net.window, net.sinks, [41, 41], 16, do)
    for name, t in zip(("dq", "dk", "dv"), grads):
        lu.check(lm_step._movable(t), w[name], w["s_" + name], net.compute, name)
