"""Plain 64-bit forms of the operators that generate text: rotation and norm of heads, a cache in pages (its layout and its 4-bit format written out element by
element), and the draw of a token in integers.  Posits are decoded and rounded by the oracle, as in lm_util."""
import math

import numpy as np
import torch

import lm_util as lu

U = lu.U


# ---- heads ----

def angles(pos, freq):
    """(cos, sin) [rows][pairs], and by how much they may be off: the fraction of a turn is taken from a product in 64 bits, then cosine and sine in 32."""
    a = np.asarray(pos, np.float64)[:, None] * np.asarray(freq, np.float64)[None, :]
    return np.cos(a), np.sin(a), 8 * U + np.abs(a) * 2.0 ** -50


def pairs(d, rot, neighbours):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if neighbours else (i, i + rot // 2)


def turn(t, cos, sin, rot, neighbours):
    """t [rows][heads][d]; the first rot elements rotated."""
    first, second = pairs(t.shape[2], rot, neighbours)
    y = t.copy()
    c, s = cos[:, None], sin[:, None]
    y[..., first] = t[..., first] * c - t[..., second] * s
    y[..., second] = t[..., second] * c + t[..., first] * s
    return y


def turn_slack(t, off, rot, neighbours):
    """How far turn() may be off where cosines and sines are by `off`, and each product and sum is rounded."""
    first, second = pairs(t.shape[2], rot, neighbours)
    s = np.zeros_like(t)
    both = (np.abs(t[..., first]) + np.abs(t[..., second])) * (off[:, None] + 3 * U)
    s[..., first] = both
    s[..., second] = both
    return s


def norm(x, w, eps):
    """(t, xhat, rstd)."""
    with np.errstate(all="ignore"):
        rstd = 1.0 / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps)
        return x * w * rstd, x * rstd, rstd


# ---- the cache ----

CACHES = ["p8", "p8_1", "p8_2", "bf16", "f4"]
MAGS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def f4_encode(x):
    """(codes, powers + 127) of x [..., d]: nearest value by distance, ties to the even code; the power as the smallest that leaves the largest at 7 or below."""
    d = x.shape[-1]
    codes, powers = np.zeros(x.shape, np.int64), np.zeros(x.shape[:-1] + (-(-d // 32),), np.int64)
    for g in range(powers.shape[-1]):
        y = x[..., 32 * g:32 * g + 32]
        top = np.abs(y).max(axis=-1)
        bad = ~np.isfinite(top)
        e = np.full(top.shape, -124)
        for k in range(-124, 125):
            e = np.where(np.where(bad, 0, top) > 7 * 2.0 ** k, k + 1, e)
        a = np.where(bad[..., None], 0, np.abs(y)) / 2.0 ** e[..., None]
        dist = np.abs(a[..., None] - MAGS)
        near = dist.min(axis=-1, keepdims=True)
        c = np.where(dist == near, np.arange(8), 99)
        even = np.where((c % 2 == 0), c, 99).min(axis=-1)
        c = np.where(even < 99, even, c.min(axis=-1))
        c = c + 8 * np.signbit(y)
        codes[..., 32 * g:32 * g + 32] = np.where(bad[..., None], 0, c)
        powers[..., g] = np.where(bad, 255, e + 127)
    return codes, powers


def f4_decode(codes, powers):
    v = np.where(codes & 8, -1, 1) * MAGS[codes & 7]
    p = np.repeat(powers, 32, axis=-1)[..., :codes.shape[-1]]
    return np.where(p == 255, np.nan, v * 2.0 ** (np.minimum(p, 254) - 127.0))


class Cache:
    """A cache as the header lays it out, as raw arrays on the host and tensors on the device."""

    def __init__(self, rng, pages, heads, page, d, fmt, junk=True):
        import paper_2105_00053_amd as pn
        self.heads, self.page, self.d, self.fmt, self.blocks = heads, page, d, fmt, -(-d // 32)
        self.tensors = pn.posit_cache_pages(pages, heads, page, d, fmt)
        self.shape = tuple(self.tensors[0].shape)
        if junk:  # whatever an unused place holds, NaN among it
            self.raw = [rng.integers(0, 65536 if fmt == "bf16" else 256, self.shape) for _ in range(2)]
            self.upload()
        else:
            self.raw = [np.zeros(self.shape, np.int64) for _ in range(2)]

    def upload(self):
        for t, r in zip(self.tensors, self.raw):
            t.view(torch.int16 if self.fmt == "bf16" else torch.uint8).copy_(torch.from_numpy(r.astype(np.uint16).view(np.int16) if self.fmt == "bf16" else r.astype(np.uint8)))

    def download(self):
        return [t.view(torch.int16 if self.fmt == "bf16" else torch.uint8).cpu().numpy().astype(np.int64) & (0xFFFF if self.fmt == "bf16" else 0xFF) for t in self.tensors]

    def element(self, values, at, d):
        return ((at // 4) * (self.d // 8) + d // 8) * 32 + (at % 4) * 8 + d % 8 if values else at * self.d + d

    def power(self, values, at, g):
        return self.page * self.d // 2 + (((at // 4) * self.blocks + g) * 4 + at % 4 if values else at * self.blocks + g)

    def put(self, which, page, at, x):
        """x [heads][d] in 64 bits, rounded, to a place of keys (0) or values (1)."""
        r, els = self.raw[which][page], [self.element(which == 1, at, d) for d in range(self.d)]
        if self.fmt == "f4":
            codes, powers = f4_encode(x)
            for d, e in enumerate(els):
                shift = 4 * (e & 1)
                r[:, e // 2] = (r[:, e // 2] & ~(15 << shift)) | codes[:, d] << shift
            for g in range(self.blocks):
                r[:, self.power(which == 1, at, g)] = powers[:, g]
        elif self.fmt == "bf16":
            r[:, els] = torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).view(torch.int16).numpy().astype(np.int64) & 0xFFFF
        else:
            from oracle import fast
            r[:, els] = np.asarray(fast.round_from_float(np.ascontiguousarray(x, np.float64).reshape(-1), self.fmt)).reshape(x.shape)

    def get(self, which, page, at):
        """[heads][d] in 64 bits."""
        r, els = self.raw[which][page], [self.element(which == 1, at, d) for d in range(self.d)]
        if self.fmt == "f4":
            codes = np.stack([r[:, e // 2] >> (4 * (e & 1)) & 15 for e in els], axis=-1)
            return f4_decode(codes, np.stack([r[:, self.power(which == 1, at, g)] for g in range(self.blocks)], axis=-1))
        if self.fmt == "bf16":
            return torch.from_numpy(r[:, els].astype(np.uint16).view(np.int16)).view(torch.bfloat16).double().numpy()
        from oracle import fast
        v = np.asarray(fast.to_float(r[:, els].astype(np.uint8).reshape(-1), self.fmt)).reshape(self.heads, self.d)
        return v.astype(np.float64)


def tables(rng, lens, page, spare=2, columns=None):
    """(table [b][columns] with pages in no order and -1 behind a sequence's end, number of pages)."""
    need = [-(-n // page) for n in lens]
    order = rng.permutation(sum(need) + spare)
    columns = max(need + [1]) if columns is None else columns
    t, first = np.full((len(lens), columns), -1, np.int32), 0
    for i, n in enumerate(need):
        t[i, :n] = order[first:first + n]
        first += n
    return t, len(order)


def dev(a, dtype=None):
    return None if a is None else torch.from_numpy(np.array(a, dtype)).cuda()


# ---- the draw ----

def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob, kept) of one row in integers.  u, temperature, top_p and min_p are binary32 values; fractions of sums are taken exactly."""
    from fractions import Fraction
    z = np.asarray(z, np.float64)
    if np.isnan(z).any() or np.isposinf(z).any() or not temperature >= 0:
        return -1, math.nan, 0
    order = [int(i) for i in np.lexsort((np.arange(len(z)), -z)) if z[i] > -np.inf]
    if not order:
        return -1, -math.inf, 0
    bits = 0
    while 1 << bits < len(z):
        bits += 1
    s = min(51, 62 - bits)
    m = z[order[0]]
    with np.errstate(all="ignore"):
        e = [1.0 if temperature == 0 else math.exp((z[i] - m) * (1.0 / float(temperature))) for i in order]
    w = [int(np.rint(x * 2.0 ** s)) for x in e]
    n = len(order) if top_k <= 0 else min(top_k, len(order))
    n = 1 if temperature == 0 else n
    if top_p < 1:
        limit, before, total = Fraction(max(float(top_p), 0.0)), 0, sum(w[:n])
        keep = 0
        for i in range(n):
            if i and not before < limit * total:
                break
            keep, before = i + 1, before + w[i]
        n = keep
    least = 0.0 if math.isnan(min_p) else min(max(float(min_p), 0.0), 1.0)
    while n > 1 and e[n - 1] < least:
        n -= 1
    total = sum(w[:n])
    u = 0.0 if not u > 0 else min(float(u), float(np.nextafter(np.float32(1), np.float32(0))))
    target, up = Fraction(u) * total, 0
    for i in range(n):
        up += w[i]
        if up > target:
            break
    lp = 0.0 if temperature == 0 else (z[order[i]] - m) / float(temperature) - math.log(total / 2.0 ** s)
    return order[i], lp, n
