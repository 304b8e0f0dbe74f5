"""Plain 64-bit forms of the language-model operators, and how far a result may be from them.

Posits are decoded and rounded by the oracle.  A result of an output format is right if it lies between the roundings of value - slack and
value + slack, where `slack` is the error bound of the binary32 computation (rounding is monotone); slack is worked out for each test from
the number of roundings, U = 2^-24 each."""
import numpy as np
import torch

from oracle import fast

U = 2.0 ** -24
POSITS = ["p8", "p8_1", "p8_2", "p10_1", "p10_2", "p12_1", "p12_2", "p16"]
BITS = {"p8": 8, "p8_1": 8, "p8_2": 8, "p10_1": 10, "p10_2": 10, "p12_1": 12, "p12_2": 12, "p16": 16}


def to_format(x, fmt):
    """float array -> device tensor of `fmt`."""
    x = np.ascontiguousarray(x, dtype=np.float32)
    if fmt == "f32":
        return torch.from_numpy(x).cuda()
    if fmt == "bf16":
        return torch.from_numpy(x).to(torch.bfloat16).cuda()
    p = np.asarray(fast.round_from_float(x.reshape(-1), fmt)).reshape(x.shape)
    return torch.from_numpy(p if p.dtype == np.uint8 else p.view(np.int16)).cuda()


def values(t, fmt):
    """device tensor of `fmt` -> float64 array."""
    c = t.detach().cpu()
    if fmt in ("f32", "bf16"):
        return c.float().numpy().astype(np.float64)
    a = c.contiguous().view(torch.uint8 if BITS[fmt] == 8 else torch.int16).numpy()
    a = a if BITS[fmt] == 8 else a.view(np.uint16)
    return np.asarray(fast.to_float(a.reshape(-1).copy(), fmt)).reshape(a.shape).astype(np.float64)


def rounded(x, fmt):
    """float64 array -> the values that `fmt` rounds it to (float64)."""
    if fmt == "f32":
        return np.asarray(x, np.float32).astype(np.float64)
    if fmt == "bf16":
        return torch.from_numpy(np.asarray(x, np.float64)).to(torch.bfloat16).double().numpy()
    x = np.ascontiguousarray(x, np.float64)
    p = np.asarray(fast.round_from_float(x.reshape(-1), fmt))
    return np.asarray(fast.to_float(p, fmt)).reshape(x.shape).astype(np.float64)


def check(got, want, slack, fmt, what=""):
    """got: device tensor of `fmt`; want, slack: float64 arrays.  NaN wants NaN; infinities want themselves in float formats."""
    g = values(got, fmt)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    want = np.asarray(want, np.float64)
    slack = np.broadcast_to(np.asarray(slack, np.float64), want.shape)
    nan = np.isnan(want) | (np.isinf(want) if fmt not in ("f32", "bf16") else False)
    assert np.array_equal(np.isnan(g), nan), (what, "NaN at", np.argwhere(np.isnan(g) != nan)[:4].tolist())
    fin = np.isfinite(want)
    same = ~fin & ~nan
    assert np.array_equal(g[same], want[same]), (what, "infinities")
    w, s = np.where(fin, want, 0.0), np.where(fin, slack, 0.0)
    lo, hi = rounded(w - s, fmt), rounded(w + s, fmt)
    bad = fin & ~((g >= lo) & (g <= hi))
    if bad.any():
        at = tuple(np.argwhere(bad)[0])
        raise AssertionError("%s: %d of %d out of bounds, first at %s: got %r, want %r +- %r" % (what, bad.sum(), bad.size, at, g[at], want[at], slack[at]))


def normal(rng, shape, sigma=1.0):
    return (rng.standard_normal(shape) * sigma).astype(np.float32)


# ---- RMS norm ----

def norm_fwd(x, res, w, eps, fres):
    """(h, rstd, t) in 64 bits; h as stored."""
    h = x if res is None else rounded((x.astype(np.float32) + res.astype(np.float32)).astype(np.float64), fres)
    with np.errstate(all="ignore"):
        rstd = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
    return h, rstd, h * w


def norm_bwd(dy, h, w, rstd, dres):
    """(dx, dw, slack of dx, slack of dw)."""
    rows, cols = h.shape
    g, r = dy * w, rstd[:, None]
    c = (g * h).mean(axis=1, keepdims=True)
    dx = r * g - r ** 3 * c * h + (0 if dres is None else dres)
    k = (cols / 64 + 32) * U
    sx = k * (np.abs(r * g) + np.abs(r ** 3 * h) * np.abs(g * h).mean(axis=1, keepdims=True) + (0 if dres is None else np.abs(dres))) + 1e-37
    return dx, (dy * h * r).sum(axis=0), sx, (rows + 32) * U * np.abs(dy * h * r).sum(axis=0) + 1e-37


# ---- attention ----

def visible(n, lq, lk, window, sinks):
    """[lq][lk] truth values for a sequence of n keys."""
    p = np.arange(n - lq, n)[:, None]
    j = np.arange(lk)[None, :]
    see = (j <= p) & (j < n)
    if window:
        see &= (j > p - window) | (j < sinks)
    return see


def attention(q, k, v, scale, window, sinks, lens, bits, do=None, bits_back=16):
    """q [b][i][h][d], k and v [b][j][h'][d] in float64 -> dict of outputs and "s_" + name slacks.  `bits`: significant bits that the probabilities
    keep in the second product.  Only what a query sees enters."""
    b, lq, hq, d = q.shape
    lk, hkv = k.shape[1:3]
    z = lambda *s: np.zeros(s)  # noqa: E731
    r = {"o": z(b, lq, hq, d), "lse": np.full((b, hq, lq), -np.inf), "dq": z(b, lq, hq, d), "dk": z(b, lk, hkv, d), "dv": z(b, lk, hkv, d)}
    r.update({"s_" + n: np.zeros_like(a) for n, a in list(r.items())})
    r["s_lse"][:] = 0
    for x in range(b):
        n = max(0, min(lk, int(lens[x])))
        see = visible(n, lq, lk, window, sinks)
        for h in range(hq):
            g = h // (hq // hkv)
            for i in range(lq):
                js = np.nonzero(see[i])[0]
                if not len(js):
                    continue
                with np.errstate(all="ignore"):
                    kk, vv, qq = k[x, js, g], v[x, js, g], q[x, i, h]
                    s = scale * (kk @ qq)
                    ds = abs(scale) * (d + 4) * U * (np.abs(kk) @ np.abs(qq)) + 4 * U * np.abs(s) + 1e-30
                    m = s.max()
                    # exp's argument is taken in binary32: its rounding is relative to s and to m
                    ds = ds + 4 * U * (np.abs(s) + abs(m))
                    e = np.exp(s - m)
                    p = e / e.sum()
                    r["lse"][x, h, i] = m + np.log(e.sum())
                    dsm = ds.max() if np.isfinite(ds).all() else 0.0
                    kn = (len(js) / 4 + 64) * U
                    r["s_lse"][x, h, i] = dsm + kn + 4 * U * abs(r["lse"][x, h, i]) if np.isfinite(m) else 0
                    pr = 2 * dsm + kn + 2.0 ** -bits
                    # a probability of zero takes nothing from an infinite value that it sees only if it is zero in truth: not for finite s
                    ov = p @ vv
                    if not np.isfinite(vv).all():
                        for c in range(d):
                            col = vv[:, c]
                            if np.isnan(col).any() or (np.isposinf(col).any() and np.isneginf(col).any()):
                                ov[c] = np.nan
                            elif np.isinf(col).any():
                                ov[c] = col[np.isinf(col)][0]
                        if np.isnan(s).any():
                            ov[:] = np.nan
                    r["o"][x, i, h] = ov
                    so = pr * (p @ np.abs(np.where(np.isfinite(vv), vv, 0))) + 1e-30
                    r["s_o"][x, i, h] = so
                    if do is None:
                        continue
                    gg = do[x, i, h]
                    back = 2.0 ** -bits_back
                    dp = vv @ gg
                    ddp = (d + 4) * U * (np.abs(vv) @ np.abs(gg))
                    dd = gg @ ov
                    ddd = np.abs(gg) @ so + (d + 4) * U * (np.abs(gg) @ np.abs(ov))
                    dz = p * (dp - dd) * scale
                    ddz = abs(scale) * p * ((2 * dsm + kn + back) * (np.abs(dp) + abs(dd)) + ddp + ddd) + 1e-30
                    r["dq"][x, i, h] = dz @ kk
                    r["s_dq"][x, i, h] = ddz @ np.abs(kk) + kn * (np.abs(dz) @ np.abs(kk)) + 1e-30
                    r["dk"][x, js, g] += dz[:, None] * qq
                    r["s_dk"][x, js, g] += (ddz + (lq * (hq // hkv) / 4 + 64) * U * np.abs(dz))[:, None] * np.abs(qq) + 1e-30
                    r["dv"][x, js, g] += p[:, None] * gg
                    r["s_dv"][x, js, g] += ((2 * dsm + kn + back + (lq * (hq // hkv) / 4 + 64) * U) * p)[:, None] * np.abs(gg) + 1e-30
    return r


# ---- log probabilities ----

def logprob(z, targets, tau, top):
    """dict of logprob, lse, entropy, top_logprob, top_index, p and the slack of a log probability, one row at a time, in 64 bits."""
    rows, vocab = z.shape
    r = {"logprob": np.zeros(rows), "lse": np.zeros(rows), "entropy": np.zeros(rows), "top_logprob": np.full((rows, top), -np.inf),
         "top_index": np.full((rows, top), -1), "lp": np.zeros((rows, vocab)), "slack": np.zeros(rows), "s_entropy": np.zeros(rows)}
    for i in range(rows):
        s = tau * z[i]
        y = None if targets is None else int(targets[i])
        if np.isnan(s).any() or np.isposinf(s).any():
            for n in ("logprob", "lse", "entropy", "top_logprob", "lp"):
                r[n][i] = np.nan
            continue
        if np.isneginf(s).all():
            r["lse"][i], r["lp"][i] = -np.inf, -np.inf
            r["logprob"][i] = 0.0 if y is None or y < 0 else (-np.inf if y < vocab else np.nan)
            continue
        m = s.max()
        lse = m + np.log(np.exp(s - m).sum())
        lp = s - lse
        p = np.exp(lp)
        r["lse"][i], r["lp"][i] = lse, lp
        r["entropy"][i] = -(p[p > 0] * lp[p > 0]).sum()
        fin = np.abs(s[np.isfinite(s)])
        # each term's exponent carries the rounding of tau * z - m, the sum that of its additions
        r["slack"][i] = (vocab / 256 + 48) * U + 4 * U * (abs(m) + abs(lse)) + 4 * U * (p[np.isfinite(s)] @ (fin + abs(m)))
        r["s_entropy"][i] = (vocab / 256 + 48) * U * (1 + r["entropy"][i]) + 8 * U * (p[np.isfinite(s)] @ ((fin + abs(m)) * (1 + np.abs(lp[np.isfinite(s)]))))
        if y is not None and y >= 0:
            r["logprob"][i] = lp[y] if y < vocab else np.nan
        order = np.lexsort((np.arange(vocab), -z[i]))[:top]
        order = order[np.isfinite(z[i][order])]
        r["top_index"][i, :len(order)], r["top_logprob"][i, :len(order)] = order, lp[order]
    return r
