"""Attention of a few new tokens over a cache in pages against 64-bit forms of what the pages hold."""
import numpy as np
import pytest
import torch

import generate_util as gu
import lm_util as lu
import paper_2105_00053_amd as pn

pytestmark = pytest.mark.gpu


def fill(rng, lens, hkv, d, page, fc, junk=True, columns=None):
    """(cache whose sequences hold normal values, table, dense values of keys and values of each sequence)."""
    table, pages = gu.tables(rng, lens, page, columns=columns)
    cache = gu.Cache(rng, pages, hkv, page, d, fc, junk)
    dense = [[np.zeros((n, hkv, d)) for n in lens] for _ in range(2)]
    for b, n in enumerate(lens):
        for j in range(n):
            for which in range(2):
                cache.put(which, table[b, j // page], j % page, rng.standard_normal((hkv, d)))
                dense[which][b][j] = cache.get(which, table[b, j // page], j % page)
    cache.upload()
    return cache, table, dense


def compare(q, fq, dense, lens, new, starts, o, lse, fout, window, sinks, scale):
    qv = lu.values(q, fq)
    for b, n in enumerate(lens):
        rows = slice(int(starts[b]), int(starts[b] + new[b]))
        if new[b] == 0:
            continue
        hkv, d = dense[0][b].shape[1:]
        k, v = (x[b][None] if n else np.zeros((1, 1, hkv, d)) for x in dense)
        r = lu.attention(qv[rows][None], k, v, scale, window, sinks, [n], 16)
        lu.check(o[rows], r["o"][0], r["s_o"][0], fout, "o of %d" % b)
        lu.check(lse[rows], r["lse"][0].T, r["s_lse"][0].T, "f32", "lse of %d" % b)


@pytest.mark.parametrize("lens,new,hq,hkv,d,page,window,sinks,fq,fc,fout", [
    ([1], [1], 1, 1, 8, 16, 0, 0, "bf16", "p8", "f32"),
    ([1, 16, 17, 0, 33], [1, 1, 1, 1, 1], 4, 2, 64, 16, 0, 0, "bf16", "p8_1", "bf16"),
    ([100, 31, 250], [1, 1, 1], 8, 2, 128, 64, 0, 0, "bf16", "f4", "f32"),
    ([100, 32, 65], [3, 0, 5], 6, 2, 80, 16, 0, 0, "p8_1", "f4", "p8_1"),
    ([130, 7], [4, 7], 5, 1, 96, 32, 40, 2, "p8_2", "f4", "bf16"),
    ([130, 70], [1, 1], 20, 1, 40, 16, 33, 5, "p12_2", "f4", "f32"),
    ([90, 5], [17, 2], 4, 4, 32, 16, 0, 0, "p8", "f4", "p16"),
    ([90, 64], [1, 2], 4, 4, 96, 16, 20, 0, "bf16", "p8_2", "bf16"),
    ([77, 140], [2, 9], 8, 2, 48, 32, 0, 0, "p10_1", "bf16", "f32"),
    ([300], [1], 3, 1, 128, 256, 64, 4, "bf16", "bf16", "bf16"),
    ([60], [1], 33, 1, 128, 16, 0, 0, "bf16", "p8_1", "f32"),
    ([3, 40], [8, 1], 2, 1, 64, 16, 0, 0, "bf16", "f4", "f32"),          # more new rows than tokens
])
def test_rows_over_pages(lens, new, hq, hkv, d, page, window, sinks, fq, fc, fout):
    rng = np.random.default_rng(sum(lens) + d)
    cache, table, dense = fill(rng, lens, hkv, d, page, fc)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q = lu.to_format(lu.normal(rng, (sum(new), hq, d), 1.5), fq)
    single = all(n == 1 for n in new)
    scale = float(np.float32(0.7 / d ** 0.5))
    o, lse = pn.posit_attention_paged(q, *cache.tensors, gu.dev(table), gu.dev(lens, np.int32), fq, fc, fout, starts=None if single else gu.dev(starts), most=max(new), scale=scale,
                                      window=window, sinks=sinks)
    compare(q, fq, dense, lens, new, starts, o, lse, fout, window, sinks, scale)


@pytest.mark.parametrize("fc", ["f4", "p8_2", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_caches_in_parts(fc, d):
    """Sequences split over workgroups and ones that are not, in one call; a window and sinks on the same cache; negative and zero scales."""
    rng = np.random.default_rng(d)
    lens, new, hkv = [3001, 517, 40, 1200], [2, 1, 1, 2], 1
    cache, table, dense = fill(rng, lens, hkv, d, 32, fc, junk=False)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q = lu.to_format(lu.normal(rng, (sum(new), 3, d), 1.5), "bf16")
    for window, sinks, scale in ((0, 0, 0.1), (700, 3, 0.1), (64, 0, -0.1), (0, 0, 0.0)):
        scale = float(np.float32(scale))
        o, lse = pn.posit_attention_paged(q, *cache.tensors, gu.dev(table), gu.dev(lens, np.int32), "bf16", fc, "f32", starts=gu.dev(starts), most=2, scale=scale, window=window, sinks=sinks)
        compare(q, "bf16", dense, lens, new, starts, o, lse, "f32", window, sinks, scale)


def test_lengths_are_bounded_and_rows_of_no_sequence_stay():
    rng = np.random.default_rng(3)
    cache, table, dense = fill(rng, [64, 64], 1, 32, 16, "p8_1", columns=4)
    q = lu.to_format(lu.normal(rng, (9, 2, 32)), "bf16")
    starts = gu.dev([2, 4, 7], np.int32)
    args = (q, *cache.tensors, gu.dev(table))
    # a length beyond the table, a negative one
    o, lse = pn.posit_attention_paged(*args, gu.dev([1000, -3], np.int32), "bf16", "p8_1", "f32", starts=starts, most=3)
    full, _ = pn.posit_attention_paged(*args, gu.dev([64, 0], np.int32), "bf16", "p8_1", "f32", starts=starts, most=3)
    assert torch.equal(o[2:7], full[2:7]) and not o[4:7].any() and torch.isinf(lse[4:7]).all()
    cut, _ = pn.posit_attention_paged(*args, gu.dev([64, 0], np.int32), "bf16", "p8_1", "f32", starts=starts, most=3, longest=50)
    want, _ = pn.posit_attention_paged(*args, gu.dev([50, 0], np.int32), "bf16", "p8_1", "f32", starts=starts, most=3)
    assert torch.equal(cut[2:7], want[2:7])
    # rows in front of the first sequence, behind the last, and beyond `most`, through the C call on buffers of ones
    import ctypes
    from paper_2105_00053_amd import generate
    desc, kc, vc, tp, lp, sp = generate._cache(*cache.tensors, args[3], gu.dev([64, 64], np.int32), starts, 3, 1, 32, 9)
    lens = gu.dev([64, 64], np.int32)
    desc.HQ, desc.ql, desc.qh, desc.most, desc.longest, desc.scale = 2, 64, 32, 2, 64, 0.125
    out, stat = torch.full((9, 2, 32), 7.0, device="cuda"), torch.full((9, 2), 7.0, device="cuda")
    need = pn.posit_attention_paged_workspace(desc)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    assert generate._load().posit_attention_paged(generate._stream(), 102, 3, 100, ctypes.byref(desc), q.data_ptr(), starts.data_ptr(), lens.data_ptr(), args[3].data_ptr(),
                                                  kc, vc, out.data_ptr(), stat.data_ptr(), work.data_ptr(), need) == 0
    torch.cuda.synchronize()
    for r in (0, 1, 6, 7, 8):
        assert (out[r] == 7).all() and (stat[r] == 7).all(), r
    assert not (out[2:6] == 7).any()


@pytest.mark.parametrize("fc", ["f4", "p8_1", "bf16"])
def test_bad_pages_and_special_values_reach_only_the_rows_that_see_them(fc):
    rng = np.random.default_rng(6)
    lens, d, page = [150, 150, 150, 150], 64, 16
    cache, table, dense = fill(rng, lens, 1, d, page, fc)
    q = lu.to_format(lu.normal(rng, (4, 2, d)), "bf16")
    call = lambda table, **how: pn.posit_attention_paged(q, *cache.tensors, gu.dev(table), gu.dev(lens, np.int32), "bf16", fc, "f32", scale=0.1, **how)  # noqa: E731
    clean, clean_lse = call(table)
    near, near_lse = call(table, window=40)
    bad = table.copy()
    bad[1, 2], bad[2, 3] = -7, 10 ** 6
    o, lse = call(bad)
    assert torch.isnan(o[1:3]).all() and torch.isnan(lse[1:3]).all()
    assert torch.equal(o[0], clean[0]) and torch.equal(o[3], clean[3])
    o, lse = call(bad, window=40)     # keys 110 and up
    assert torch.equal(o, near) and torch.equal(lse, near_lse)
    # a NaN among the keys of sequence 0 (token 20), among the values of sequence 3 (token 21, element 5)
    special = np.zeros((1, d))
    special[0, 5] = np.nan
    for which, b, j in ((0, 0, 20), (1, 3, 21)):
        was = cache.get(which, table[b, j // page], j % page).copy()
        cache.put(which, table[b, j // page], j % page, np.where(np.isnan(special), special, was))
    cache.upload()
    o, lse = call(table)
    assert torch.isnan(o[0]).all() and torch.isnan(lse[0]).all()
    gone = torch.zeros(d, dtype=torch.bool, device="cuda")
    gone[:32 if fc == "f4" else 0] = True
    gone[5] = True
    assert torch.isnan(o[3][:, gone]).all() and torch.equal(lse[3], clean_lse[3])
    torch.testing.assert_close(o[3][:, ~gone], clean[3][:, ~gone], rtol=1e-5, atol=1e-6)
    assert torch.equal(o[1:3], clean[1:3])
    o, lse = call(table, window=40)
    assert torch.equal(o, near) and torch.equal(lse, near_lse)
    if fc == "bf16":  # an infinity among the values
        cache.put(1, table[3, 21 // page], 21 % page, np.where(np.isnan(special), -np.inf, was))
        cache.upload()
        assert torch.isneginf(call(table)[0][3][:, 5]).all()


def test_an_append_then_attention_is_attention_over_dense_rows():
    """The same patterns through posit_attention_fwd, keys and values dense, within both calls' roundings of probabilities to 16 bits."""
    rng = np.random.default_rng(12)
    b, l, hq, hkv, d, page = 3, 70, 4, 2, 64, 16
    x = lu.to_format(lu.normal(rng, (b * l, hq + 2 * hkv, d), 1.5), "p8_2")
    table, pages = gu.tables(rng, [l] * b, page)
    k, v = pn.posit_cache_pages(pages, hkv, page, d, "p8_2")
    lens, starts, freq = gu.dev([l] * b, np.int32), gu.dev(np.arange(b + 1) * l, np.int32), pn.rope_frequencies(d)
    q = pn.posit_cache_append(x[:, hq:hq + hkv], x[:, hq + hkv:], k, v, gu.dev(table), lens, "p8_2", "p8_2", starts=starts, q=x[:, :hq], fq="p8_2", inv_freq=freq)
    dense = pn.posit_cache_read(k, v, gu.dev(table), lens, l, d, "p8_2", "p8_2")
    want, want_lse, _ = pn.posit_attention_fwd(q.view(b, l, hq, d), *dense, "p8_2", "p8_2", "f32")
    o, lse = pn.posit_attention_paged(q, k, v, gu.dev(table), lens, "p8_2", "p8_2", "f32", starts=starts, most=l)
    torch.testing.assert_close(o.view(b, l, hq, d), want, rtol=0, atol=2.0 ** -14 * 64)
    torch.testing.assert_close(lse.view(b, l, hq).transpose(1, 2), want_lse, rtol=2e-6, atol=2e-6)


def test_offsets_beyond_32_bits():
    """A cache of more than 4 GiB a tensor: the last pages hold what the first ones would."""
    rng = np.random.default_rng(13)
    hkv, d, page, n = 1, 128, 4096, 200
    pages = 9000
    k, v = (torch.zeros((pages, hkv, page * d), dtype=torch.uint8, device="cuda") for _ in range(2))
    assert k.numel() > 2 ** 32
    x = lu.to_format(lu.normal(rng, (2 * n, 2, d)), "p8_1")
    table = gu.dev([[pages - 1], [0]], np.int32)
    lens, starts = gu.dev([n, n], np.int32), gu.dev([0, n, 2 * n], np.int32)
    x[n:] = x[:n]
    pn.posit_cache_append(x[:, :1], x[:, 1:], k, v, table, lens, "p8_1", "p8_1", starts=starts)
    assert torch.equal(k[pages - 1], k[0]) and torch.equal(v[pages - 1], v[0]) and k[0].any() and v[0].any()
    q = lu.to_format(lu.normal(rng, (2, 4, d)), "bf16")
    q[1] = q[0]
    o, _ = pn.posit_attention_paged(q, k, v, table, lens, "bf16", "p8_1", "f32", longest=n)
    assert torch.equal(o[0], o[1]) and o.any()
    dense, _ = pn.posit_cache_read(k, v, table, lens, n, d, "p8_1", "f32")
    assert torch.equal(dense[0], dense[1])
