"""Infinities and NaN all over values and back-propagated errors: which results they reach, in blocks that a wave's rows see alike and at the mask's edges,
and what they may cost."""
import numpy as np
import pytest
import torch

import paper_2105_00053_amd as pn
from lm_util import attention, check, normal, to_format, values

pytestmark = pytest.mark.gpu

INF = float("inf")


def _sprinkle(t, rng, share):
    """A share of the elements of a bfloat16 tensor becomes +inf, -inf or NaN; whole stretches stay as they are."""
    kind = rng.integers(0, 3, t.shape)
    at = (rng.random(t.shape) < share) & (rng.random((t.shape[0], t.shape[1], 1, 1)) < 0.5)
    for k, v in enumerate((INF, -INF, float("nan"))):
        t[torch.from_numpy(at & (kind == k)).cuda()] = v


def _inputs(seed, b, lq, lk, hq, hkv, d):
    rng = np.random.default_rng([seed, b, lq, lk, hq, d])
    shapes = ((b, lq, hq, d), (b, lk, hkv, d), (b, lk, hkv, d), (b, lq, hq, d))
    return (rng,) + tuple(to_format(normal(rng, s), "bf16") for s in shapes)


@pytest.mark.parametrize("lq,lk,hq,hkv,d", [(200, 300, 2, 1, 64), (300, 300, 3, 1, 40), (130, 260, 2, 2, 96), (140, 140, 5, 1, 128), (1, 700, 4, 1, 64), (5, 420, 3, 1, 128),
                                            (1, 333, 2, 1, 40), (2, 300, 2, 2, 72)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 0), (70, 40), (33, 3), (9, 200)])
def test_values_that_are_not_finite(lq, lk, hq, hkv, d, window, sinks):
    for share in (1e-3, 0.2):
        rng, q, k, v, _ = _inputs(1, 2, lq, lk, hq, hkv, d)
        _sprinkle(v, rng, share)
        lens = [lk, lk - 41]
        o, lse, copy = pn.posit_attention_fwd(q, k, v, "bf16", "bf16", "bf16", window=window, sinks=sinks, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), fcopy="f32")
        w = attention(values(q, "bf16"), values(k, "bf16"), values(v, "bf16"), np.float64(np.float32(1 / np.sqrt(d))), window, sinks, lens, 16)
        check(copy, w["o"], w["s_o"], "f32", "o_copy")
        check(o, w["o"], w["s_o"], "bf16", "o")
        check(lse, w["lse"], w["s_lse"], "f32", "lse")


@pytest.mark.parametrize("l,hq,hkv,d", [(200, 2, 1, 64), (100, 1, 1, 128), (150, 3, 1, 40), (260, 1, 1, 96), (90, 40, 1, 16)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 40), (33, 3), (9, 150)])
def test_errors_that_are_not_finite(l, hq, hkv, d, window, sinks):
    """dV = P^T dO: an infinity in dO reaches the keys that its row sees."""
    for share in (1e-3, 0.2):
        rng, q, k, v, do = _inputs(2, 1, l, l, hq, hkv, d)
        o, lse, copy = pn.posit_attention_fwd(q, k, v, "bf16", "bf16", "f32", window=window, sinks=sinks)
        _sprinkle(do, rng, share)
        dv = pn.posit_attention_bwd(do, q, k, v, o, lse, "bf16", "bf16", "bf16", "f32", "f32", window=window, sinks=sinks)[2]
        w = attention(values(q, "bf16"), values(k, "bf16"), values(v, "bf16"), np.float64(np.float32(1 / np.sqrt(d))), window, sinks, [l], 16, values(do, "bf16"))
        check(dv, w["dv"], w["s_dv"], "f32", "dv")


def _time(call):
    """Least of five, in us."""
    call()
    best = INF
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b) * 1e3)
    return best


@pytest.mark.parametrize("pass_,window,sinks", [("prompt", 0, 0), ("prompt", 600, 4), ("token", 0, 0), ("token", 4096, 4), ("backward", 0, 0), ("backward", 600, 4)])
def test_a_diverged_step_takes_about_as_long(pass_, window, sinks):
    """With a NaR in every key's value (every row's error): a wave reads what is noted of a block, a load for each 64 blocks, and walks 32 rows of the blocks at
    its edges, some hundred loads in series of a microsecond at most; the kernel for few queries reads the values a second time."""
    b, l, hq, hkv, d = (64, 8192, 8, 1, 64) if pass_ == "token" else (1, 8192, 4, 1, 64)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    lq = 1 if pass_ == "token" else l
    q, k, v, do = (pn.posit_round(torch.randn(s, generator=g, device="cuda"), "p8_1") for s in ((b, lq, hq, d), (b, l, hkv, d), (b, l, hkv, d), (b, lq, hq, d)))
    how = {"window": window, "sinks": sinks}
    o, lse, copy = pn.posit_attention_fwd(q, k, v, "p8_1", "p8_1", "bf16", fcopy="f32", **how)

    def call():
        if pass_ == "backward":
            return pn.posit_attention_bwd(do, q, k, v, copy, lse, "p8_1", "p8_1", "p8_1", "f32", "bf16", **how)
        return pn.posit_attention_fwd(q, k, v, "p8_1", "p8_1", "bf16", **how)

    clean = _time(call)
    (do if pass_ == "backward" else v)[:, :, :, 17] = 128
    diverged = _time(call)
    print("%s, window %d: %.0f us, with NaR %.0f" % (pass_, window, clean, diverged))
    assert diverged < 4 * clean + 1000
    out = call()[2 if pass_ == "backward" else 0]
    nan = torch.isnan(out.float())
    assert nan[..., 17].all() and not nan[..., 18:].any() and not nan[..., :17].any()
