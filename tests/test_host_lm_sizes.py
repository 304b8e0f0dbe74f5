"""Sizes at the ends of what the language-model entry points accept (nothing is launched)."""
import ctypes
import os

import pytest

MOST = 2 ** 63 - 1


@pytest.fixture(scope="module")
def L():
    from paper_2105_00053_amd import build, lm
    if not os.path.exists(build.LIB):
        build.build()
    return lm._load()


@pytest.mark.parametrize("b,lq,hq,hkv,d", [(4, 1, 32, 8, 128), (1, 1, 8, 2, 64), (2, 5, 4, 1, 40)])
def test_windows_and_sinks_beyond_the_cache_plan_as_none(L, b, lq, hq, hkv, d):
    """A window of all keys or more is none, and sinks beyond the cache are all keys: the parts of a cache, and so the workspace, are the same."""
    from paper_2105_00053_amd import AttentionDesc

    def need(window, sinks, which=0, lk=4096):
        return L.posit_attention_workspace(which, 3, ctypes.byref(AttentionDesc(b, hq, hkv, lq, lk, d, window, sinks, 0.125, *[1] * 9)))

    whole = need(0, 0)
    assert whole > 0
    for window in (4096, 5000, 2 ** 31, 2 ** 62, MOST - 4096, MOST):
        for sinks in (0, 4, 4096, 2 ** 40, MOST):
            assert need(window, sinks) == whole, (window, sinks)
            assert need(window, sinks, which=1) == need(0, 0, which=1)
    for sinks in (4096, 2 ** 33, MOST - 200, MOST):
        assert need(100, sinks) == whole, sinks
    assert need(100, 4) < whole  # a short window does plan for fewer keys


def test_attention_of_more_workgroups_than_a_launch_counts_is_refused(L):
    """A launch of 2^32 threads or more would leave workgroups out without an error."""
    from paper_2105_00053_amd import AttentionDesc
    at, none = ctypes.c_void_p(0x1000), ctypes.c_void_p(0)  # never dereferenced

    def fwd(**kw):
        d = AttentionDesc(**dict(dict(D=8, window=0, sinks=0, scale=1.0), **kw))
        return L.posit_attention_fwd(none, 3, 3, 102, ctypes.byref(d), at, at, at, none, at, at, 0, none, at, 1 << 60), L.posit_attention_workspace(0, 3, ctypes.byref(d))

    def bwd(**kw):
        d = AttentionDesc(**dict(dict(D=8, window=0, sinks=0, scale=1.0), **kw))
        return L.posit_attention_bwd(none, 3, 3, 3, 100, 102, ctypes.byref(d), *[at] * 4, none, *[at] * 6, 1 << 60), L.posit_attention_workspace(1, 3, ctypes.byref(d))

    many = dict(B=16000, HQ=60000, HKV=3000)
    assert fwd(LQ=1, LK=0, **many) == bwd(LQ=1, LK=0, **many) == bwd(LQ=0, LK=1, **many) == (2, 0)
    long = dict(B=1, HQ=1, HKV=1)
    assert fwd(LQ=100, LK=2 ** 30, **long) == bwd(LQ=1, LK=2 ** 30, **long) == bwd(LQ=2 ** 30, LK=1, **long) == (2, 0)
