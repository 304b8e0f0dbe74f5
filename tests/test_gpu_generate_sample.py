"""The draw of a token against the same in integers.  A weight's last bit may differ by one unit (exp in 64 bits is right to one): among these seeds no number falls that close to a border,
which has a chance of some 2^-30 for each."""
import math

import numpy as np
import pytest
import torch

import generate_util as gu
import lm_util as lu
import paper_2105_00053_amd as pn

pytestmark = pytest.mark.gpu

ONE = float(np.nextafter(np.float32(1), np.float32(0)))


def run(z, fmt, u, temperature=None, top_k=None, top_p=None, min_p=None):
    t = lu.to_format(z, fmt)
    f = lambda a, kind: None if a is None else gu.dev(np.broadcast_to(np.asarray(a, kind), (len(z),)), kind)  # noqa: E731
    got = pn.posit_sample(t, f(u, np.float32), fmt, temperature=f(temperature, np.float32), top_k=f(top_k, np.int32), top_p=f(top_p, np.float32), min_p=f(min_p, np.float32))
    return [x.cpu().numpy() for x in got], lu.values(t, fmt)


def check(z, fmt, u, **how):
    (token, logprob, kept), v = run(z, fmt, u, **how)
    at = lambda name, r, none: none if how.get(name) is None else np.broadcast_to(np.asarray(how[name], np.float32 if name != "top_k" else np.int32), (len(z),))[r].item()  # noqa: E731
    u = np.broadcast_to(np.asarray(u, np.float32), (len(z),))
    for r in range(len(z)):
        want = gu.sample(v[r], u[r].item(), at("temperature", r, 1.0), at("top_k", r, 0), at("top_p", r, 1.0), at("min_p", r, 0.0))
        assert (token[r], kept[r]) == (want[0], want[2]), (r, token[r], kept[r], want)
        if math.isnan(want[1]):
            assert math.isnan(logprob[r])
        else:
            assert logprob[r] == want[1] or abs(logprob[r] - want[1]) <= 4 * lu.U * (1 + abs(want[1])), (r, logprob[r], want)


@pytest.mark.parametrize("fmt", ["p8", "p8_1", "p8_2", "p10_1", "p10_2", "p12_1", "p12_2", "p16", "bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 500, 3001, 20011])
def test_formats_and_sizes(fmt, vocab):
    rng = np.random.default_rng(vocab)
    rows = 6
    z = lu.normal(rng, (rows, vocab), 2.5)
    u = rng.random(rows).astype(np.float32)
    check(z, fmt, u)
    check(z, fmt, u, temperature=0.7, top_k=max(1, vocab // 3), top_p=0.9, min_p=0.01)
    check(z, fmt, u, temperature=[0, 1, 0.3, 5, 100, 1e-3], top_k=[0, 1, 5, vocab, vocab + 7, -3], top_p=[1, 0.5, 0.99, 0.2, 1.5, 0.7], min_p=[0, 0.1, 0.5, 1e-4, 0.9, 0])


@pytest.mark.parametrize("fmt", ["p16", "f32", "p8_2"])
@pytest.mark.parametrize("how", [dict(top_k=40), dict(top_k=1), dict(top_p=0.95), dict(top_p=0.01), dict(min_p=0.05), dict(temperature=0.0), dict(top_k=1000, top_p=0.999)])
def test_limits_alone(fmt, how):
    rng = np.random.default_rng(3)
    check(lu.normal(rng, (5, 9001), 2.0), fmt, rng.random(5).astype(np.float32), **how)


def test_long_rows():
    rng = np.random.default_rng(4)
    for fmt, vocab in (("p16", 131072), ("f32", 65537), ("bf16", 140001), ("p8_1", 300007)):
        check(lu.normal(rng, (2, vocab), 2.0), fmt, np.array([0.3, 0.999], np.float32), temperature=[0.8, 1.0], top_p=[0.9, 1.0])


def test_ends_of_the_random_numbers():
    z = np.array([[0, 1, 1, -1, 1]] * 7, np.float32)
    u = np.array([0, ONE, 1.0, 2.0, -1.0, np.nan, 1e-40], np.float32)
    (token, _, kept), _ = run(z, "f32", u)
    assert token.tolist() == [1, 3, 3, 3, 1, 1, 1] and (kept == 5).all()


def test_equal_logits_are_drawn_by_their_indices():
    """Of n equal weights the draw takes floor(u n): 2^s is a multiple of every power of two here."""
    n = 4096
    u = np.array([0, 0.25, 0.5, 0.75, 1 / 4096, 1 / 4096 - 2.0 ** -30, ONE], np.float32)
    (token, logprob, kept), _ = run(np.zeros((7, n), np.float32), "f32", u)
    assert token.tolist() == [0, 1024, 2048, 3 * 1024, 1, 0, 4095] and (kept == n).all()
    assert np.allclose(logprob, -np.log(n), rtol=1e-7)
    for k, p, want in ((3, 1.0, 3), (0, 0.5, 2048), (0, 0.50001, 2049), (100, 0.25, 25), (1, 0.0, 1), (0, 0.0, 1), (0, -1.0, 1), (0, np.nan, n)):
        (_, _, kept), _ = run(np.zeros((1, n), np.float32), "f32", [0.0], top_k=k, top_p=p)
        assert kept[0] == want, (k, p, kept)


def test_shares_follow_the_weights():
    """Over all u = (i + 1/2) / n, each token is drawn as often as its share says, to one of n."""
    z = np.array([2.0, -1.0, 0.5, 2.0, -30.0], np.float32)
    n = 2000
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    (token, logprob, _), _ = run(np.tile(z, (n, 1)), "f32", u, temperature=0.9)
    p = np.exp((z - 2.0) / 0.9)
    p /= p.sum()
    counts = np.bincount(token, minlength=5)
    assert (np.abs(counts - n * p) <= 1.01).all()
    assert np.allclose(np.exp(logprob), p[token], rtol=1e-5)


def test_special_rows():
    inf, nan = np.inf, np.nan
    z = np.array([[1, nan, 2], [1, inf, 2], [-inf, -inf, -inf], [-inf, 3, -inf], [-0.0, 0.0, -0.0], [3e38, -3e38, 1]], np.float32)
    for fmt in ("f32", "bf16"):
        check(z, fmt, 0.6)
    (token, logprob, kept), _ = run(z, "f32", 0.6)
    assert token.tolist()[:4] == [-1, -1, -1, 1] and kept.tolist()[:4] == [0, 0, 0, 1] and np.isneginf(logprob[2]) and logprob[3] == 0
    (token, logprob, kept), _ = run(z[3:], "f32", 0.6, temperature=[-1.0, nan, inf])
    assert token.tolist()[:2] == [-1, -1] and np.isnan(logprob[:2]).all() and token[2] == 2 and kept[2] == 3  # without a difference left, by index: 0, 1, 2 of shares 1/3 in falling order 0, 2, 1
    t = lu.to_format(np.array([[1, nan, 2], [1, 0, 2]], np.float32), "p16")
    token, _, _ = pn.posit_sample(t, gu.dev([0.0, 0.0], np.float32), "p16")
    assert token.tolist() == [-1, 2]
    (token, _, kept), _ = run(z[4:], "f32", 0.9, min_p=[nan, 2.0])
    assert kept.tolist() == [3, 1]


def test_views_and_empty_batches():
    rng = np.random.default_rng(5)
    wide = lu.to_format(lu.normal(rng, (4, 1000), 2.0), "p16")
    u = gu.dev(rng.random(4), np.float32)
    for first, n in ((0, 999), (1, 501), (3, 8)):
        part = wide[:, first:first + n]
        a, b = pn.posit_sample(part, u, "p16", top_p=u), pn.posit_sample(part.contiguous(), u, "p16", top_p=u)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    token, logprob, kept = pn.posit_sample(wide[:0], u[:0], "p16")
    assert token.shape == logprob.shape == kept.shape == (0,)
    with pytest.raises(pn.PositError):
        pn.posit_sample(wide[:, :0], u, "p16")
    with pytest.raises(pn.PositError):
        pn.posit_sample(wide, u[:3], "p16")
    with pytest.raises(pn.PositError):
        pn.posit_sample(wide, u, "p16", top_k=u)
