"""Norms of queries and keys with the rotation by positions, forward and backward, against 64-bit forms; gradients against differences, too."""
import numpy as np
import pytest
import torch

import generate_util as gu
import lm_util as lu
import paper_2105_00053_amd as pn

pytestmark = pytest.mark.gpu
U = lu.U


def make(rng, t, hq, hkv, d, fx):
    """(views of q and k in the rows of one product, their values)."""
    x = lu.to_format(lu.normal(rng, (t, hq + 2 * hkv, d), 1.5), fx)
    v = lu.values(x, fx)
    return (x[:, :hq], v[:, :hq]), (x[:, hq:hq + hkv], v[:, hq:hq + hkv])


def forward(x, w, cos, sin, off, rot, neighbours, eps):
    """(y, its slack, xhat, rstd): sums of d squares and a root and a division in binary32."""
    k = (x.shape[2] / 4 + 24) * U
    if w is None:
        t, hat, rstd = x, x, None
        k = 0.0
    else:
        t, hat, rstd = gu.norm(x, w, eps)
    if cos is None:
        return t, k * np.abs(t), hat, rstd
    return gu.turn(t, cos, sin, rot, neighbours), gu.turn_slack(t, off + k, rot, neighbours) + k * np.abs(t), hat, rstd


@pytest.mark.parametrize("t,hq,hkv,d,rot,neighbours,fx,fw,fy", [
    (1, 1, 1, 8, 8, False, "p8", "f32", "f32"),
    (5, 4, 2, 64, 64, False, "p8_1", "p16", "p8_1"),
    (33, 5, 1, 80, 40, False, "p8_2", "p12_2", "bf16"),
    (33, 4, 4, 96, 96, True, "bf16", "f32", "bf16"),
    (7, 8, 2, 128, 128, False, "p16", "bf16", "p12_1"),
    (300, 3, 1, 128, 64, True, "f32", "f32", "f32"),
    (9, 2, 1, 256, 256, False, "p12_2", "p10_1", "p10_2"),
    (9, 2, 2, 200, 72, True, "p10_2", "p8", "p16"),
    (4, 3, 1, 30, 30, False, "p8_2", "p16", "f32"),      # runs of pairs that end inside four
    (4, 3, 1, 30, 14, False, "bf16", "p16", "p8"),
    (4, 3, 1, 22, 10, True, "p16", "p16", "p16"),
    (6, 3, 2, 2, 2, False, "f32", "f32", "f32"),
    (2500, 4, 2, 64, 64, False, "p8_2", "p16", "f32"),   # more rows than workgroups
    (9001, 1, 1, 24, 16, False, "p8_1", "f32", "bf16"),  # workgroups with more than one block, values from a table
    (4099, 2, 1, 8, 8, True, "p8", "bf16", "p8"),
])
@pytest.mark.parametrize("how", ["both", "norm", "turn", "none"])
def test_forward_and_backward(t, hq, hkv, d, rot, neighbours, fx, fw, fy, how):
    rng = np.random.default_rng(t + d)
    (q, qv), (k, kv) = make(rng, t, hq, hkv, d, fx)
    norm, turns = how in ("both", "norm"), how in ("both", "turn")
    w = [lu.to_format(1 + lu.normal(rng, (d,), 0.2), fw) if norm else None for _ in range(2)]
    wv = [lu.values(a, fw) if norm else None for a in w]
    pos = rng.integers(-5000, 200000, t).astype(np.int32)
    freq = pn.rope_frequencies(rot)
    cos, sin, off = gu.angles(pos, freq.cpu().numpy()) if turns else (None, None, 0.0)
    args = dict(positions=gu.dev(pos) if turns else None, inv_freq=freq if turns else None, wq=w[0], wk=w[1], fw=fw, neighbours=neighbours)
    eps = float(np.float32(1e-6))
    yq, yk, rstd = pn.posit_qk_norm_rope_fwd(q, k, fx, fy, eps=1e-6, **args)
    fd = fx if t % 2 and fx != "f32" else "bf16"
    g = [lu.to_format(lu.normal(rng, v.shape), fd) for v in (qv, kv)]
    dq, dk, dwq, dwk = pn.posit_qk_norm_rope_bwd(g[0], g[1], q, k, rstd, fd, fx, fy, fdw="f32", **args)
    assert (rstd is None) == (not norm) and (dwq is None) == (dwk is None) == (not norm)
    for n, (x, y, dx, dw, gr) in enumerate(((qv, yq, dq, dwq, g[0]), (kv, yk, dk, dwk, g[1]))):
        want, slack, hat, r = forward(x, wv[n], cos, sin, off, rot, neighbours, eps)
        lu.check(y, want, slack + 1e-37, fy, "y%d" % n)
        gv = lu.values(gr, fd)
        gt, gs = (gu.turn(gv, cos, -sin, rot, neighbours), gu.turn_slack(gv, off, rot, neighbours)) if turns else (gv, 0 * gv)
        if not norm:
            lu.check(dx, gt, gs + 1e-37, fy, "dx%d" % n)
            continue
        lu.check(rstd[:, n * hq:n * hq + x.shape[1]], r[..., 0], (d / 4 + 24) * U * r[..., 0], "f32", "rstd%d" % n)
        c = (d / 4 + 48) * U
        gw, mean = gt * wv[n], lambda a: a.mean(axis=2, keepdims=True)
        want = r * (gw - hat * mean(gw * hat))
        slack = r * (gs * np.abs(wv[n]) + np.abs(hat) * mean(gs * np.abs(wv[n] * hat))) + c * r * (np.abs(gw) + np.abs(hat) * mean(np.abs(gw * hat)))
        lu.check(dx, want, slack + 1e-37, fy, "dx%d" % n)
        terms = gt * hat
        lu.check(dw, terms.sum(axis=(0, 1)), (gs * np.abs(hat)).sum(axis=(0, 1)) + (d / 4 + 24 + t * x.shape[1] / 8 + 64) * U * np.abs(terms).sum(axis=(0, 1)) + 1e-37, "f32", "dw%d" % n)


def test_without_keys_rows_or_heads():
    rng = np.random.default_rng(1)
    (q, qv), _ = make(rng, 3, 2, 1, 16, "p8_1")
    w, freq, pos = lu.to_format(np.ones(16, np.float32), "f32"), pn.rope_frequencies(16), torch.arange(3, dtype=torch.int32, device="cuda")
    y, none, rstd = pn.posit_qk_norm_rope_fwd(q, None, "p8_1", "f32", positions=pos, inv_freq=freq, wq=w, fw="f32")
    assert none is None and rstd.shape == (3, 2)
    both = pn.posit_qk_norm_rope_fwd(q, q[:, :1], "p8_1", "f32", positions=pos, inv_freq=freq, wq=w, wk=w, fw="f32")
    assert torch.equal(both[0], y) and torch.equal(both[1], y[:, :1]) and torch.equal(both[2][:, :2], rstd)
    dq, dk, dwq, dwk = pn.posit_qk_norm_rope_bwd(y, None, q, None, rstd, "f32", "p8_1", "f32", positions=pos, inv_freq=freq, wq=w, fw="f32")
    assert dk is None and dwk is None and dwq.shape == (16,)
    e = q[:0]
    y, _, rstd = pn.posit_qk_norm_rope_fwd(e, e, "p8_1", "f32", positions=pos[:0], inv_freq=freq, wq=w, wk=w, fw="f32")
    assert y.shape == (0, 2, 16)
    _, _, dwq, dwk = pn.posit_qk_norm_rope_bwd(y, y, e, e, rstd, "f32", "p8_1", "f32", positions=pos[:0], inv_freq=freq, wq=w, wk=w, fw="f32")
    assert not dwq.any() and not dwk.any()
    with pytest.raises(pn.PositError):
        pn.posit_qk_norm_rope_fwd(q, None, "p8_1", "f32", positions=pos)
    with pytest.raises(pn.PositError):
        pn.posit_qk_norm_rope_fwd(q, q, "p8_1", "f32", wq=w, fw="f32")
    with pytest.raises(pn.PositError):
        pn.posit_qk_norm_rope_fwd(q, None, "p8_1", "f32", positions=pos, inv_freq=pn.rope_frequencies(18))


def test_far_positions_turn_by_the_fraction():
    """At the largest position the product's rounding in 64 bits is 2^31 2^-53 of a turn's radians: far below binary32's own."""
    pos = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7, 0], np.int32)
    x = np.zeros((4, 1, 64), np.float32)
    x[..., :32] = 1
    freq = pn.rope_frequencies(64)
    y, _, _ = pn.posit_qk_norm_rope_fwd(torch.from_numpy(x).cuda(), None, "f32", "f32", positions=gu.dev(pos), inv_freq=freq)
    # exact products as integers times the frequencies' own fractions
    from fractions import Fraction
    two_pi = Fraction(314159265358979323846264338327950288419716939937510, 10 ** 50) * 2
    for r, p in enumerate(pos.tolist()):
        for i, f in enumerate(freq.cpu().numpy().tolist()):
            turns = Fraction(f) * p / two_pi
            a = float((turns - round(turns)) * two_pi)
            bound = 8 * U + abs(f * p) * 2.0 ** -50
            assert abs(y[r, 0, i].item() - np.cos(a)) < bound and abs(y[r, 0, 32 + i].item() - np.sin(a)) < bound


def test_special_values_stay_in_their_head():
    rng = np.random.default_rng(4)
    x = lu.normal(rng, (6, 3, 32))
    x[1, 2, 5], x[4, 0, 31] = np.nan, np.inf
    t = lu.to_format(x, "bf16")
    w, freq, pos = lu.to_format(np.ones(32, np.float32), "f32"), pn.rope_frequencies(32), torch.arange(6, dtype=torch.int32, device="cuda")
    y, _, rstd = pn.posit_qk_norm_rope_fwd(t, None, "bf16", "p8_2", positions=pos, inv_freq=freq, wq=w, fw="f32")
    v = lu.values(y, "p8_2")
    clean = np.ones((6, 3), bool)
    clean[1, 2] = clean[4, 0] = False
    assert np.isnan(v[1, 2]).all() and np.isnan(v[4, 0]).any() and np.isfinite(v[clean]).all()
    assert torch.isnan(rstd[1, 2]) and rstd[4, 0] == 0
    zero = torch.zeros((2, 1, 32), device="cuda")
    y, _, rstd = pn.posit_qk_norm_rope_fwd(zero, None, "f32", "f32", positions=pos[:2], inv_freq=freq, wq=w, fw="f32")
    assert not y.any() and torch.allclose(rstd, torch.full_like(rstd, 1e3))


@pytest.mark.parametrize("neighbours", [False, True])
def test_gradients_by_differences(neighbours):
    """d (sum of y times g) by a step of 2^-6 either way in 64 bits, from the forward call's own outputs in binary32: their rounding (some 2^-20 of the sum of magnitudes) over the
    step, and the third derivative's share, some 2^-12 of values of order one."""
    rng = np.random.default_rng(5)
    t, h, d, rot = 2, 2, 16, 12
    x, g = rng.standard_normal((t, h, d)), rng.standard_normal((t, h, d))
    w = 1 + 0.2 * rng.standard_normal(d)
    pos, freq = torch.tensor([3, 40], dtype=torch.int32, device="cuda"), pn.rope_frequencies(rot)
    f32 = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()  # noqa: E731
    how = dict(positions=pos, inv_freq=freq, fw="f32", neighbours=neighbours)
    run = lambda x, w: pn.posit_qk_norm_rope_fwd(f32(x), None, "f32", "f32", eps=0.01, wq=f32(w), **how)  # noqa: E731
    total = lambda x, w: float((run(x, w)[0].double().cpu().numpy() * np.asarray(g, np.float32)).sum())  # noqa: E731
    dx, _, dw, _ = pn.posit_qk_norm_rope_bwd(f32(g), None, f32(x), None, run(x, w)[2], "f32", "f32", "f32", wq=f32(w), **how)
    step = 2.0 ** -6
    for at in [(0, 0, 0), (0, 1, 5), (1, 0, 11), (1, 1, 13), (0, 0, 15)]:
        e = np.zeros_like(x)
        e[at] = step
        assert abs((total(x + e, w) - total(x - e, w)) / (2 * step) - dx[at].item()) < 0.01
    for i in (0, 6, 11, 14):
        e = np.zeros(d)
        e[i] = step
        assert abs((total(x, w + e) - total(x, w - e)) / (2 * step) - dw[i].item()) < 0.01


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("d, rot", [(48, 16), (48, 36), (50, 18)])
def test_what_is_not_rotated_stays(d, rot, neighbours):
    """Elements from `rot` on are the given ones, whatever stands beside them: infinities and NaN reach no other element there, and no rotated one."""
    rng = np.random.default_rng(d + rot)
    x = lu.normal(rng, (9, 4, d))
    x[2, 1, rot:] = np.where(np.arange(d - rot) % 3 == 0, np.inf, x[2, 1, rot:])
    x[5, 3, d - 1], x[6, 0, rot + 1] = np.nan, -np.inf
    t, pos, freq = lu.to_format(x, "f32"), torch.arange(3, 12, dtype=torch.int32, device="cuda"), pn.rope_frequencies(rot)
    how = dict(positions=pos, inv_freq=freq, neighbours=neighbours)
    outs = list(pn.posit_qk_norm_rope_fwd(t[:, :3], t[:, 3:], "f32", "f32", **how)[:2])
    outs += pn.posit_qk_norm_rope_bwd(t[:, :3], t[:, 3:], t[:, :3], t[:, 3:], None, "f32", "f32", "f32", **how)[:2]
    got = [torch.cat(outs[:2], 1), torch.cat(outs[2:], 1)]
    if d % 8 == 0:
        k, v = pn.posit_cache_pages(1, 4, 16, d, "bf16")
        table, lens, starts = gu.dev(np.array([[0]], np.int32)), gu.dev(np.array([12], np.int32)), gu.dev(np.array([0, 9], np.int32))
        got.append(pn.posit_cache_append(t, t, k, v, table, lens, "f32", "bf16", starts=starts, q=t, fq="f32", inv_freq=freq, neighbours=neighbours))
        dense = pn.posit_cache_read(k, v, table, lens, 12, d, "bf16", "f32")[0][0, 3:]
        want = lu.values(lu.to_format(x, "bf16"), "bf16")
        assert np.array_equal(dense[..., rot:].cpu().numpy(), want[..., rot:], equal_nan=True) and torch.isfinite(dense[..., :rot]).all()
    for y in got:
        assert np.array_equal(y[..., rot:].cpu().numpy(), x[..., rot:], equal_nan=True) and torch.isfinite(y[..., :rot]).all()
