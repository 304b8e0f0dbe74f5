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
