"""Log probabilities of given tokens, entropy, top alternatives and the gradient, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2105_00053_amd as pn
from lm_util import POSITS, U, check, logprob, normal, to_format, values

pytestmark = pytest.mark.gpu

INF = float("inf")


def _run(z, targets, fmt, tau, top):
    zt = z if isinstance(z, torch.Tensor) else to_format(z, fmt)
    tt = None if targets is None else torch.from_numpy(np.asarray(targets, np.int32)).cuda()
    return zt, tt, pn.posit_token_logprob_fwd(zt, tt, fmt, inv_temperature=tau, top=top)


def _forward(z, targets, fmt, tau=1.0, top=0):
    zt, tt, (lp, lse, ent, tlp, tix) = _run(z, targets, fmt, tau, top)
    want = logprob(values(zt, fmt), targets, np.float64(np.float32(tau)), top)
    s = want["slack"]
    check(lse, want["lse"], s, "f32", "lse")
    check(ent, want["entropy"], want["s_entropy"], "f32", "entropy")
    if targets is not None:
        check(lp, want["logprob"], s + 4 * U * np.abs(np.where(np.isfinite(want["logprob"]), want["logprob"], 0)), "f32", "logprob")
    if top:
        assert np.array_equal(tix.cpu().numpy(), want["top_index"])
        check(tlp, want["top_logprob"], s[:, None] + 4 * U * np.abs(np.where(np.isfinite(want["top_logprob"]), want["top_logprob"], 0)), "f32", "top")
    return zt, tt, lse, ent, want


@pytest.mark.parametrize("rows,vocab", [(1, 1), (2, 2), (3, 5), (1, 63), (2, 64), (3, 65), (1, 255), (2, 513), (1, 2048), (5, 2049), (2, 4099), (1, 20003), (3, 70001), (300, 130), (1100, 37)])
def test_forward_over_sizes(rows, vocab):
    rng = np.random.default_rng([1, rows, vocab])
    for fmt, top in (("p16", 5), ("p8_2", 20), ("f32", 1), ("bf16", 64), ("p12_2", 0)):
        _forward(normal(rng, (rows, vocab), 2), rng.integers(0, vocab, rows), fmt, top=top)


@pytest.mark.parametrize("fmt", POSITS + ["bf16", "f32"])
def test_formats_temperatures_and_gradients(fmt):
    rng = np.random.default_rng(2)
    for tau in (1.0, 0.37, 8.0):
        rows, vocab = 6, 777
        y = rng.integers(0, vocab, rows)
        y[2], y[4] = -1, vocab
        zt, tt, lse, ent, want = _forward(normal(rng, (rows, vocab), 1.5), y, fmt, tau, 7)
        g1, g2 = normal(rng, rows), normal(rng, rows, 0.3)
        _gradients(zt, tt, lse, ent, want, y, g1, g2, fmt, tau)


def _gradients(zt, tt, lse, ent, want, y, g1, g2, fmt, tau, formats=("f32", "bf16", "p8_2", "p16")):
    t32 = np.float64(np.float32(tau))
    vocab = want["lp"].shape[1]
    for a, b in ((g1, g2), (g1, None), (None, g2)):
        with np.errstate(all="ignore"):
            lp = want["lp"]
            p = np.exp(lp)
            hit = np.zeros_like(p)
            ga = np.zeros(len(p)) if a is None else a.astype(np.float64)
            for i, t in enumerate(y):
                if a is not None and t < 0:
                    ga[i] = 0
                elif a is not None and t >= vocab:
                    ga[i] = np.nan
                elif a is not None:
                    hit[i, t] = 1
            d = ga[:, None] * (hit - p)
            # a probability carries the error of its log; the term of the entropy also that of the log and of the entropy itself
            e = (want["slack"] + 8 * U)[:, None] + 4 * U * np.abs(np.where(np.isfinite(lp), lp, 0))
            s = np.abs(ga)[:, None] * (p * e + 2 * U)
            if b is not None:
                term = np.where(p > 0, p * (lp + want["entropy"][:, None]), 0)
                d = d - b[:, None].astype(np.float64) * term
                s = s + np.abs(b)[:, None] * p * (e * (2 + np.abs(np.where(p > 0, lp, 0)) + want["entropy"][:, None]) + want["s_entropy"][:, None])
            d, s = t32 * d, t32 * (s + 2 * U * np.abs(d)) + 1e-37
        for fg in formats:
            got = pn.posit_token_logprob_bwd(zt, tt if a is not None else None, lse, ent, None if a is None else torch.from_numpy(a).cuda(),
                                             None if b is None else torch.from_numpy(b).cuda(), fmt, fg, inv_temperature=tau)
            check(got, d, s, fg, "dlogits %s" % fg)


@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 7), (2, 64), (5, 1001), (1, 40001), (513, 129)])
def test_gradient_over_sizes(rows, vocab):
    rng = np.random.default_rng([3, rows, vocab])
    y = rng.integers(0, vocab, rows)
    for fmt in ("p16", "p8_2", "f32"):
        zt, tt, lse, ent, want = _forward(normal(rng, (rows, vocab), 2), y, fmt)
        _gradients(zt, tt, lse, ent, want, y, normal(rng, rows), normal(rng, rows, 0.2), fmt, 1.0, formats=("f32", "bf16"))


def test_gradient_against_differences():
    rng = np.random.default_rng(4)
    z, y, tau = normal(rng, (2, 30), 1.0), [4, 29], 0.7
    zt, tt, (lp, lse, ent, _, _) = _run(z, y, "f32", tau, 0)
    g1, g2 = np.float32([0.5, -1.5]), np.float32([2.0, 0.25])
    got = values(pn.posit_token_logprob_bwd(zt, tt, lse, ent, torch.from_numpy(g1).cuda(), torch.from_numpy(g2).cuda(), "f32", "f32", inv_temperature=tau), "f32")

    def loss(v):
        w = logprob(v, y, np.float64(np.float32(tau)), 0)
        return (g1 * w["logprob"] + g2 * w["entropy"]).sum()

    for r in range(2):
        for c in (0, 4, 17, 29):
            d = np.zeros((2, 30))
            d[r, c] = 1e-5
            v = z.astype(np.float64)
            assert abs((loss(v + d) - loss(v - d)) / 2e-5 - got[r, c]) < 1e-5


@pytest.mark.parametrize("vocab", [5, 600, 5003, 33000])
@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_masked_logits(vocab, fmt):
    """-inf and the lowest finite value in masked places, rows that keep one token, rows that keep none."""
    rng = np.random.default_rng([5, vocab])
    z = normal(rng, (7, vocab), 2)
    z[0, rng.random(vocab) < 0.7] = -INF
    z[1] = -INF
    z[2] = -INF
    z[2, vocab // 2] = 1.5
    z[3, : vocab - 1] = -3.3895313892515355e38
    z[4] = -3.3895313892515355e38
    z[5, vocab - 1] = -INF
    y = np.array([vocab - 1, 0, vocab // 2, vocab - 1, 3, 1, 2])
    zt, tt, lse, ent, want = _forward(z, y, fmt, top=min(vocab, 9))
    _gradients(zt, tt, lse, ent, want, y, normal(rng, 7), normal(rng, 7, 0.2), fmt, 1.0, formats=("f32", "p8_2"))


def test_not_a_number_stays_in_its_row():
    rng = np.random.default_rng(6)
    z = normal(rng, (5, 3001), 2)
    z[1, 2900], z[3, 17], z[4, 0] = np.nan, INF, -INF
    y = np.array([0, 1, 2, 3, 4])
    for fmt in ("f32", "bf16", "p16"):
        zz = z.copy()
        if fmt == "p16":
            zz[4, 0] = 0  # a posit has no -inf: it would be NaR
        zt, tt, lse, ent, want = _forward(zz, y, fmt, top=4)
        _gradients(zt, tt, lse, ent, want, y, normal(rng, 5), normal(rng, 5), fmt, 1.0, formats=("f32", "p16"))


@pytest.mark.parametrize("vocab", [64, 700, 20000])
def test_ties_go_to_the_lowest_index(vocab):
    rng = np.random.default_rng([7, vocab])
    for z in (np.zeros((2, vocab), np.float32), np.repeat(normal(rng, (2, vocab // 4)), 4, axis=1), np.where(rng.random((2, vocab)) < 0.5, 0.0, -0.0).astype(np.float32),
              np.sort(normal(rng, (2, vocab)), axis=1), -np.sort(normal(rng, (2, vocab)), axis=1)):
        for fmt in ("p8", "p8_2", "f32"):
            _forward(z, [0, vocab - 1], fmt, top=64 if vocab >= 64 else vocab)
            _forward(z, None, fmt, top=3)


def test_more_alternatives_than_tokens():
    z = np.float32([[1, 3, 2]])
    _, _, (lp, lse, ent, tlp, tix) = _run(z, [1], "f32", 1.0, 6)
    assert tix.cpu().tolist() == [[1, 2, 0, -1, -1, -1]]
    assert torch.isinf(tlp[0, 3:]).all()


def test_rows_with_a_pitch_and_other_streams():
    rng = np.random.default_rng(8)
    for fmt, cols in (("p16", 5003), ("p8_2", 911), ("f32", 40001)):
        big = to_format(normal(rng, (6, cols + 9), 2), fmt)
        z = big[1:5, 3:3 + cols]
        y = torch.from_numpy(rng.integers(0, cols, 4).astype(np.int32)).cuda()
        g = torch.from_numpy(normal(rng, 4)).cuda()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            a = pn.posit_token_logprob_fwd(z, y, fmt, top=5)
            da = pn.posit_token_logprob_bwd(z, y, a[1], a[2], g, g, fmt, "bf16")
        side.synchronize()
        b = pn.posit_token_logprob_fwd(z.contiguous(), y, fmt, top=5)
        db = pn.posit_token_logprob_bwd(z.contiguous(), y, b[1], b[2], g, g, fmt, "bf16")
        # the splits of a row may depend on its address's alignment, so sums are compared within their bound
        want = logprob(values(z.contiguous(), fmt), y.cpu().numpy(), 1.0, 5)
        for r in (a, b):
            check(r[0], want["logprob"], want["slack"] + 4 * U * np.abs(want["logprob"]), "f32")
            check(r[1], want["lse"], want["slack"], "f32")
            assert np.array_equal(r[4].cpu().numpy(), want["top_index"])
        assert (da.float() - db.float()).abs().max() <= 2.0 ** -8 * g.abs().max() * 4


def test_repeats_are_identical():
    rng = np.random.default_rng(9)
    z, y = normal(rng, (3, 60001), 2), [5, 6, 7]
    first = _run(z, y, "p16", 1.0, 10)
    for _ in range(3):
        again = pn.posit_token_logprob_fwd(first[0], first[1], "p16", top=10)
        assert all(torch.equal(a, b) for a, b in zip(first[2], again))


def test_empty():
    z = torch.empty((0, 50), dtype=torch.float32, device="cuda")
    y = torch.empty((0,), dtype=torch.int32, device="cuda")
    out = pn.posit_token_logprob_fwd(z, y, "f32", top=3)
    assert out[0].shape == (0,) and out[4].shape == (0, 3)
