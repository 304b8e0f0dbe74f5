"""RMS norm with the residual's addition (forward, scaled output, backward) and rows times scales, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2105_00053_amd as pn
from lm_util import BITS, POSITS, U, check, norm_bwd, norm_fwd, normal, rounded, to_format, values
from oracle import fast

pytestmark = pytest.mark.gpu

EPS = 1e-6
SIZES = [(1, 1), (3, 7), (2, 64), (5, 65), (4, 511), (2, 512), (7, 520), (3, 1000), (2, 2047), (2, 2048), (1, 4096), (3, 5119), (1, 8192), (2, 8200), (1, 20001)]


def _inputs(rows, cols, fx, fres, fw, seed):
    rng = np.random.default_rng([seed, rows, cols])
    x, w = to_format(normal(rng, (rows, cols), 0.5), fx), to_format(1 + normal(rng, cols, 0.1), fw)
    res = None if fres is None else to_format(normal(rng, (rows, cols)) * np.where(rng.random((1, cols)) < 0.05, 6, 1), fres)
    return rng, x, res, w


def _forward(x, res, w, fx, fres, fw, fy, scaled, rows, cols):
    y, scale, out, rstd = pn.posit_rmsnorm_fwd(x, w, fx, fw, fy, eps=EPS, res=res, fres=fres, scaled=scaled)
    h, r, t = norm_fwd(values(x, fx), None if res is None else values(res, fres), values(w, fw), EPS, fres)
    k = (cols / 64 + 32) * U
    check(rstd, r, k * r, "f32", "rstd")
    if res is not None:
        assert np.array_equal(values(out, fres), h)  # one rounding of a binary32 sum: no slack
    if scaled:
        a = np.abs(t).max(axis=1)
        e = np.where(a > 0, np.floor(np.log2(np.where(a > 0, a, 1))), 2)
        check(scale, r * 2.0 ** (e - 2), k * r * 2.0 ** (e - 2), "f32", "scale")
        up = 2.0 ** (2 - e)[:, None]
        check(y, t * up, 2 * U * np.abs(t * up), fy, "patterns")
        check(pn.posit_scale_rows(y, scale, fy, "f32"), values(y, fy) * values(scale, "f32")[:, None], 2 * U * np.abs(values(y, fy) * values(scale, "f32")[:, None]), "f32", "values")
    else:
        check(y, t * r[:, None], k * np.abs(t * r[:, None]), fy, "y")
    return out if res is not None else x, rstd, h, r


@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward_and_backward_over_sizes(rows, cols):
    for fx, fres, fw, fy, scaled in (("p8_1", "p16", "p16", "p8_1", True), ("p8_2", "bf16", "p12_2", "bf16", False), ("bf16", None, "f32", "p8", True)):
        rng, x, res, w = _inputs(rows, cols, fx, fres, fw, 1)
        out, rstd, h, r = _forward(x, res, w, fx, fres, fw, fy, scaled, rows, cols)
        fh = fres or fx
        dy, dres = to_format(normal(rng, (rows, cols)), "bf16"), to_format(normal(rng, (rows, cols)), "p16")
        dx, dw = pn.posit_rmsnorm_bwd(dy, out, w, rstd, "bf16", fh, fw, "bf16", "f32", dres=dres, fdres="p16")
        wx, ww, sx, sw = norm_bwd(values(dy, "bf16"), h, values(w, fw), values(rstd, "f32"), values(dres, "p16"))
        check(dx, wx, sx, "bf16", "dx")
        check(dw, ww, sw, "f32", "dw")


@pytest.mark.parametrize("fx", POSITS + ["bf16", "f32"])
@pytest.mark.parametrize("fres", ["p8_2", "p12_1", "p16", "bf16", "f32"])
def test_forward_formats(fx, fres):
    for i, fy in enumerate(POSITS + ["bf16", "f32"]):
        _, x, res, w = _inputs(3, 333, fx, fres, "p16", 2)
        _forward(x, res, w, fx, fres, "p16", fy, i % 2 == 0, 3, 333)


@pytest.mark.parametrize("fd", ["p8_2", "p16", "bf16", "f32"])
def test_backward_formats(fd):
    for fh in ("p8", "p16", "bf16", "f32"):
        for fdx, fdw in (("p8_2", "p16"), ("p16", "p12_2"), ("f32", "bf16"), ("bf16", "f32")):
            rng, h, _, w = _inputs(37, 130, fh, None, "p12_2", 3)
            _, _, _, rstd = pn.posit_rmsnorm_fwd(h, w, fh, "p12_2", "f32", eps=EPS)
            dy = to_format(normal(rng, (37, 130)), fd)
            dx, dw = pn.posit_rmsnorm_bwd(dy, h, w, rstd, fd, fh, "p12_2", fdx, fdw)
            wx, ww, sx, sw = norm_bwd(values(dy, fd), values(h, fh), values(w, "p12_2"), values(rstd, "f32"), None)
            check(dx, wx, sx, fdx, "dx")
            check(dw, ww, sw, fdw, "dw")
    dx, dw = pn.posit_rmsnorm_bwd(dy, h, w, rstd, fd, fh, "p12_2", fdx, fdw, want_dw=False)
    assert dw is None
    check(dx, wx, sx, fdx, "dx alone")


@pytest.mark.parametrize("rows,cols", [(1025, 640), (4099, 96), (700, 2056), (2000, 300)])
def test_weight_gradient_over_many_rows(rows, cols):
    rng, h, _, w = _inputs(rows, cols, "p16", None, "p16", 4)
    _, _, _, rstd = pn.posit_rmsnorm_fwd(h, w, "p16", "p16", "bf16", eps=EPS)
    dy = to_format(normal(rng, (rows, cols)), "bf16")
    dx, dw = pn.posit_rmsnorm_bwd(dy, h, w, rstd, "bf16", "p16", "p16", "bf16", "f32")
    wx, ww, sx, sw = norm_bwd(values(dy, "bf16"), values(h, "p16"), values(w, "p16"), values(rstd, "f32"), None)
    check(dx, wx, sx, "bf16", "dx")
    check(dw, ww, sw, "f32", "dw")
    again = pn.posit_rmsnorm_bwd(dy, h, w, rstd, "bf16", "p16", "p16", "bf16", "f32")
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


def test_gradient_against_differences():
    rng, h, _, w = _inputs(4, 48, "f32", None, "f32", 5)
    hv, wv = values(h, "f32"), values(w, "f32")
    _, _, _, rstd = pn.posit_rmsnorm_fwd(h, w, "f32", "f32", "f32", eps=EPS)
    dy = to_format(normal(rng, (4, 48)), "f32")
    dx, dw = pn.posit_rmsnorm_bwd(dy, h, w, rstd, "f32", "f32", "f32", "f32", "f32")
    g = values(dy, "f32")

    def loss(hh, ww):
        return (g * hh * ww / np.sqrt((hh * hh).mean(axis=1, keepdims=True) + EPS)).sum()

    step = 1e-5
    for r, c in ((0, 0), (1, 17), (3, 47)):
        d = np.zeros_like(hv)
        d[r, c] = step
        assert abs((loss(hv + d, wv) - loss(hv - d, wv)) / (2 * step) - float(dx[r, c])) < 1e-5
    for c in (0, 31):
        d = np.zeros_like(wv)
        d[c] = step
        assert abs((loss(hv, wv + d) - loss(hv, wv - d)) / (2 * step) - float(dw[c])) < 1e-4


def test_views_with_pitches_odd_addresses_and_other_streams():
    rng = np.random.default_rng(6)
    big = [to_format(normal(rng, (9, 701)), f) for f in ("p8_1", "p16", "bf16")]
    x, res, dy = (b[1:8, 3:600] for b in big)
    w = to_format(1 + normal(rng, 598, 0.1), "p16")[1:]
    dense = [t.contiguous() for t in (x, res, dy)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for scaled in (False, True):
        with torch.cuda.stream(side):
            a = pn.posit_rmsnorm_fwd(x, w, "p8_1", "p16", "p8_2", res=res, fres="p16", scaled=scaled)
            ga = pn.posit_rmsnorm_bwd(dy, a[2], w, a[3], "bf16", "p16", "p16", "bf16", "f32", dres=dy, fdres="bf16")
        side.synchronize()
        b = pn.posit_rmsnorm_fwd(dense[0], w.clone(), "p8_1", "p16", "p8_2", res=dense[1], fres="p16", scaled=scaled)
        gb = pn.posit_rmsnorm_bwd(dense[2], b[2], w.clone(), b[3], "bf16", "p16", "p16", "bf16", "f32", dres=dense[2], fdres="bf16")
        for s, t in zip(a + ga, b + gb):
            assert (s is None and t is None) or torch.equal(s, t)


def test_residual_written_in_place():
    rng, x, res, w = _inputs(5, 777, "p8_1", "p16", "p16", 7)
    y, _, out, _ = pn.posit_rmsnorm_fwd(x, w, "p8_1", "p16", "bf16", res=res, fres="p16")
    y2 = torch.empty_like(y)
    from paper_2105_00053_amd import binding
    status = pn.lm._load().posit_rmsnorm_fwd(binding._stream(), 3, 1, 1, 102, 5, 777, x.data_ptr(), 777, res.data_ptr(), 777, w.data_ptr(), 1e-6, res.data_ptr(), 777,
                                             y2.data_ptr(), 777, None, None)
    assert status == 0
    assert torch.equal(res, out.view(torch.int16)) and torch.equal(y, y2)


def test_special_rows():
    """NaR, NaN and infinities stay in their row; rows of zeros, of the smallest and of the largest posits."""
    rng, x, res, w = _inputs(8, 200, "p16", None, "p16", 8)
    x[1, 5] = -32768  # NaR
    x[2] = 0
    x[3] = 1
    x[4] = 32767
    clean = x.clone()
    clean[1, 5] = 0
    for scaled in (False, True):
        for fy in ("p8_1", "bf16"):
            y, scale, _, rstd = pn.posit_rmsnorm_fwd(x, w, "p16", "p16", fy, eps=EPS, scaled=scaled)
            y0, scale0, _, rstd0 = pn.posit_rmsnorm_fwd(clean, w, "p16", "p16", fy, eps=EPS, scaled=scaled)
            assert np.isnan(values(y, fy)[1]).all() and torch.isnan(rstd[1])
            keep = [0, 2, 3, 4, 5, 6, 7]
            assert torch.equal(y[keep], y0[keep]) and torch.equal(rstd[keep], rstd0[keep])
            assert (values(y, fy)[2] == 0).all()
            if scaled:
                assert torch.isnan(scale[1]) and torch.equal(scale[keep], scale0[keep])
            h, r, t = norm_fwd(values(clean, "p16"), None, values(w, "p16"), EPS, None)
            assert np.isfinite(values(y, fy)[keep]).all()
            if not scaled:
                check(y0, t * r[:, None], 64 * U * np.abs(t * r[:, None]), fy)
    f = torch.from_numpy(normal(rng, (3, 70))).cuda()
    f[0, 3], f[1, 69] = float("inf"), float("nan")
    y, scale, _, _ = pn.posit_rmsnorm_fwd(f, torch.ones(70, device="cuda"), "f32", "f32", "p8", scaled=True)
    assert np.isnan(values(y, "p8")[:2]).all() and np.isfinite(values(y, "p8")[2]).all()
    assert torch.isnan(scale[:2]).all() and torch.isfinite(scale[2])


@pytest.mark.parametrize("fmt", POSITS)
def test_codec_over_every_pattern(fmt):
    """posit_scale_rows by 1 decodes every pattern exactly and rounds binary32 as the oracle does."""
    n = 1 << BITS[fmt]
    p = np.arange(n).astype(np.uint8 if BITS[fmt] == 8 else np.uint16)
    t = torch.from_numpy(p if p.dtype == np.uint8 else p.view(np.int16)).cuda().reshape(1, n)
    one = torch.ones(1, device="cuda")
    f = pn.posit_scale_rows(t, one, fmt, "f32")
    v = np.asarray(fast.to_float(p, fmt))
    assert np.array_equal(f.cpu().numpy()[0], v, equal_nan=True)
    rng = np.random.default_rng(9)
    x = np.concatenate([v, np.nextafter(v, np.float32(np.inf)), (v[:-1] + v[1:]) / 2, normal(rng, 5000) * np.exp2(rng.integers(-45, 45, 5000)),
                        [0.0, -0.0, np.inf, -np.inf, 1e-40, -1e-45, 3e38]]).astype(np.float32)
    got = pn.posit_scale_rows(torch.from_numpy(x).cuda().reshape(1, -1), one, "f32", fmt)
    want = np.asarray(fast.round_from_float(x, fmt))
    assert np.array_equal(got.cpu().view(torch.uint8 if BITS[fmt] == 8 else torch.int16).numpy()[0].view(want.dtype), want)


def test_scale_rows_sizes_and_pitches():
    rng = np.random.default_rng(10)
    for rows, cols in ((1, 1), (3, 17), (5, 256), (2, 1029), (300, 33)):
        x = to_format(normal(rng, (rows, cols + 5)), "p8_2")[:, 2:2 + cols]
        s = torch.from_numpy(np.exp2(normal(rng, rows))).cuda()
        want = values(x.contiguous(), "p8_2") * values(s, "f32")[:, None]
        for f in ("f32", "bf16", "p16", "p8_2"):
            check(pn.posit_scale_rows(x, s, "p8_2", f), want, 2 * U * np.abs(want), f)


def test_empty():
    z = torch.empty((0, 8), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(8, device="cuda")
    y, scale, out, rstd = pn.posit_rmsnorm_fwd(z, w, "bf16", "f32", "p8", scaled=True)
    assert y.shape == (0, 8) and scale.shape == (0,)
    dx, dw = pn.posit_rmsnorm_bwd(z, z, w, rstd, "bf16", "bf16", "f32", "bf16", "f32")
    assert dx.shape == (0, 8) and (dw == 0).all()
