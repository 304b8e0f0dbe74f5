"""Keys and values into and out of a cache in pages: every byte of it against the layout written out element by element.  Append computes in 64 bits, so what it stores is
the nearest to what numpy computes in 64 bits, unless that lies within some 1e-13 of a border of two patterns: not among these seeds' thousands of values."""
import numpy as np
import pytest
import torch

import generate_util as gu
import lm_util as lu
import paper_2105_00053_amd as pn

pytestmark = pytest.mark.gpu


def case(rng, new, had, hq, hkv, d, page, fx, fc, junk=True):
    """(q, k, v as views of one product's rows, cache, table, lens, starts)."""
    lens = [n + h for n, h in zip(new, had)]
    table, pages = gu.tables(rng, lens, page)
    cache = gu.Cache(rng, pages, hkv, page, d, fc, junk)
    x = lu.to_format(lu.normal(rng, (sum(new), hq + 2 * hkv, d), 1.5), fx)
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], cache, table, lens, np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


def slack_of_queries(x, want, norm, pos, freq, rot, neighbours, fq):
    """Posits are rounded from 64 bits; other queries from binary32: as posit_qk_norm_rope_fwd's, from a sum of d squares, a root, a division and a rotation."""
    if fq not in ("f32", "bf16"):
        return 1e-12 * np.abs(want) + 1e-37
    k = (x.shape[2] / 4 + 24) * lu.U if norm else 0.0
    t = np.abs(want) if not norm else np.abs(want).max(axis=2, keepdims=True) + 0 * want  # rotation keeps a pair's length
    return (k + lu.U) * np.abs(want) + (gu.turn_slack(t * 2 ** 0.5, gu.angles(pos, freq.cpu().numpy())[2] + k, rot, neighbours) if rot else 0) + 1e-37


@pytest.mark.parametrize("new,had,hq,hkv,d,rot,neighbours,norm,page,fx,fw,fq,fc", [
    ([1], [0], 1, 1, 8, 8, False, True, 16, "p8", "f32", "f32", "p8"),
    ([1, 1, 1], [0, 15, 16], 4, 2, 64, 64, False, False, 16, "p8_1", "f32", "bf16", "p8_1"),
    ([5, 0, 33, 2], [3, 9, 0, 30], 4, 2, 32, 32, False, True, 16, "p8_2", "p16", "p8_2", "p8_2"),
    ([17, 40], [47, 0], 5, 1, 80, 40, True, True, 32, "bf16", "p12_2", "bf16", "f4"),
    ([3, 70, 1], [64, 60, 127], 8, 4, 128, 128, False, True, 64, "p8_2", "f32", "bf16", "f4"),
    ([9, 20], [7, 0], 2, 2, 40, 24, False, True, 16, "p16", "bf16", "p16", "f4"),
    ([4, 30], [100, 250], 2, 1, 96, 96, True, False, 256, "f32", "f32", "p12_1", "bf16"),
    ([8, 1], [0, 3], 3, 1, 24, 0, False, True, 16, "p12_2", "p8", "p10_1", "bf16"),
    ([6], [0], 3, 1, 48, 0, False, False, 16, "p8_2", "f32", "f32", "f4"),
])
def test_append_and_read(new, had, hq, hkv, d, rot, neighbours, norm, page, fx, fw, fq, fc):
    rng = np.random.default_rng(sum(new) + d)
    q, k, v, cache, table, lens, starts = case(rng, new, had, hq, hkv, d, page, fx, fc)
    w = [lu.to_format(1 + lu.normal(rng, (d,), 0.2), fw) if norm else None for _ in range(2)]
    freq = pn.rope_frequencies(rot) if rot else None
    single = all(n == 1 for n in new)
    yq = pn.posit_cache_append(k, v, *cache.tensors, gu.dev(table), gu.dev(lens, np.int32), fx, fc, starts=None if single else gu.dev(starts), q=q, fq=fq, inv_freq=freq,
                               wq=w[0], wk=w[1], fw=fw, neighbours=neighbours)
    got = cache.download()
    pos = np.concatenate([np.arange(h, h + n) for n, h in zip(new, had)])
    out = []
    for x, ww in ((q, w[0]), (k, w[1])):
        t = lu.values(x, fx)
        if norm:
            t = gu.norm(t, lu.values(ww, fw), float(np.float32(1e-6)))[0]
        out.append(gu.turn(t, *gu.angles(pos, freq.cpu().numpy())[:2], rot, neighbours) if rot else t)
    lu.check(yq, out[0], slack_of_queries(lu.values(q, fx), out[0], norm, pos, freq, rot, neighbours, fq), fq, "q")
    values = lu.values(v, fx)
    for b in range(len(new)):
        for i in range(new[b]):
            at, r = had[b] + i, starts[b] + i
            for which, x in ((0, out[1]), (1, values)):
                cache.put(which, table[b, at // page], at % page, x[r])
    for which in range(2):
        assert np.array_equal(got[which], cache.raw[which]), (which, np.argwhere(got[which] != cache.raw[which])[:4].tolist())
    # and back; what a sequence had before is whatever the junk stands for
    longest = max(lens) + 3
    for fout in ("f32", "bf16", "p8_2"):
        dense = pn.posit_cache_read(*cache.tensors, gu.dev(table), gu.dev(lens, np.int32), longest, d, fc, fout)
        for which in range(2):
            want = np.zeros((len(new), longest, hkv, d))
            for b, n in enumerate(lens):
                for j in range(n):
                    want[b, j] = cache.get(which, table[b, j // page], j % page)
            with np.errstate(over="ignore"):  # values are binary32 on the way, where 4 times 2^127 of junk in 4 bits is infinite
                lu.check(dense[which], want.astype(np.float32), 0.0, fout, "read %d" % which)


def test_places_that_are_none_are_left_out():
    """Bad page numbers, tokens beyond the table, sequences without tokens, rows of no sequence: nothing else is written, and queries are, where a row is a sequence's."""
    rng = np.random.default_rng(8)
    cache = gu.Cache(rng, 5, 1, 16, 32, "p8_1")
    before = cache.download()
    x = lu.to_format(lu.normal(rng, (12, 3, 32)), "p8_1")
    q, k, v = x[:, :1], x[:, 1:2], x[:, 2:]
    # four rows each: page 2 then a number past the last; -1; lens below the rows; beyond the columns.  rows 11 and up are nobody's
    table = np.array([[2, 5], [-1, 3], [4, 4], [1, 0]], np.int32)
    lens = np.array([18, 3, 1, 34], np.int32)
    starts = np.array([0, 4, 7, 9, 11], np.int32)
    freq = pn.rope_frequencies(32)
    yq = pn.posit_cache_append(k, v, *cache.tensors, gu.dev(table), gu.dev(lens), "p8_1", "p8_1", starts=gu.dev(starts), q=q, fq="f32", inv_freq=freq)
    got = cache.download()
    cache.raw = before
    pos = np.concatenate([np.arange(14, 18), np.arange(0, 3), np.arange(-1, 1), np.arange(32, 34)])
    turned = gu.turn(lu.values(k, "p8_1")[:11], *gu.angles(pos, freq.cpu().numpy())[:2], 32, False)
    for r, page, at in ((0, 2, 14), (1, 2, 15), (8, 4, 0)):
        cache.put(0, page, at, turned[r])
        cache.put(1, page, at, lu.values(v, "p8_1")[r])
    for which in range(2):
        assert np.array_equal(got[which], cache.raw[which])
    x = lu.values(q, "p8_1")[:11]
    want = gu.turn(x, *gu.angles(pos, freq.cpu().numpy())[:2], 32, False)
    lu.check(yq[:11], want, slack_of_queries(x, want, False, pos, freq, 32, False, "f32"), "f32")
    dense, _ = pn.posit_cache_read(*cache.tensors, gu.dev(table), gu.dev(lens), 40, 32, "p8_1", "f32")
    d = dense.cpu().numpy()
    assert np.isfinite(d[0, 14:16]).all() and np.isnan(d[0, 16:18]).all() and np.isnan(d[1, :3]).all() and np.isnan(d[3, 32:34]).all()
    assert not d[0, 18:].any() and not d[1, 3:].any()


def test_blocks_with_special_values():
    """NaN and infinities make a block of 4 bits NaN, and one element of the other formats; the largest numbers saturate, the smallest vanish in 4 bits only."""
    x = np.zeros((4, 1, 64), np.float32)
    x[0, 0, :3] = [np.nan, 1, 2]
    x[1, 0, 40], x[1, 0, 2] = -np.inf, 3
    x[2, 0, :4] = [3.3e38, -1e38, 1.0, 2.9e38]
    x[3, 0, :4], x[3, 0, 32:36] = [1e-38, -3e-39, 1e-45, 0], [1, 0.2, 0.12, -0.13]
    t = lu.to_format(x, "f32")
    table, lens = torch.tensor([[0]], dtype=torch.int32, device="cuda"), torch.tensor([4], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    for fc in gu.CACHES:
        cache = gu.Cache(np.random.default_rng(0), 1, 1, 16, 64, fc)
        pn.posit_cache_append(t, t, *cache.tensors, table, lens, "f32", fc, starts=starts)
        got = cache.download()
        for r in range(4):
            for which in range(2):
                if fc == "f4" and r == 2:
                    want = np.where(np.arange(64) < 32, gu.f4_decode(*gu.f4_encode(np.clip(x[r].astype(np.float64), -6 * 2.0 ** 125, 6 * 2.0 ** 125))), 0)
                    cache.put(which, 0, r, want)
                    cache.raw[which][0, :, cache.power(which == 1, r, 1)] = 3
                else:
                    with np.errstate(over="ignore"):
                        cache.put(which, 0, r, x[r].astype(np.float64))
        one = lambda r: np.where((r & 0x7FFF) > 0x7F80, 0x7FC0, r) if fc == "bf16" else r  # noqa: E731  (a NaN is any of bfloat16's)
        assert np.array_equal(one(got[0]), one(cache.raw[0])) and np.array_equal(one(got[1]), one(cache.raw[1])), fc


def test_many_sequences_and_many_rows():
    """More sequences than a workgroup looks through at once, and more rows than workgroups take one by one; the keys as given, so equal to the rows' patterns."""
    rng = np.random.default_rng(9)
    b, page, d = 700, 16, 16
    new = rng.integers(0, 15, b)
    new[5] = 1500
    lens = new + rng.integers(0, 20, b)
    table, pages = gu.tables(rng, lens.tolist(), page)
    x = lu.to_format(lu.normal(rng, (int(new.sum()), 2, d)), "p8_2")
    k, v = pn.posit_cache_pages(pages, 1, page, d, "p8_2")
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    assert pn.posit_cache_append(x[:, :1], x[:, 1:], k, v, gu.dev(table), gu.dev(lens, np.int32), "p8_2", "p8_2", starts=gu.dev(starts)) is None
    dense = pn.posit_cache_read(k, v, gu.dev(table), gu.dev(lens, np.int32), int(lens.max()), d, "p8_2", "f32")
    want = torch.zeros((2, b, int(lens.max()), d))
    vals = torch.from_numpy(lu.values(x, "p8_2")).float()
    for i in range(b):
        at = slice(int(lens[i] - new[i]), int(lens[i]))
        for which in range(2):
            want[which, i, at] = vals[starts[i]:starts[i + 1], which]
    for which in range(2):
        assert torch.equal(dense[which][:, :, 0].cpu(), want[which])
