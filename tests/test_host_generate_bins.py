"""The draw's first bins of floats: what a search finds in a bin are the logits that it counts, under masks too."""
import ctypes
import os

import numpy as np
import pytest


@pytest.fixture(scope="module")
def bins():
    from paper_2105_00053_amd import build
    if not os.path.exists(build.HOSTCHECK):
        build.build()
    f = ctypes.CDLL(build.HOSTCHECK).hostcheck_sample_bins
    f.restype = None
    f.argtypes = [ctypes.c_int, ctypes.c_double, ctypes.c_int, ctypes.c_float, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]

    def run(z, temperature):
        z = np.ascontiguousarray(z, np.float32)
        out = np.empty(len(z), np.int32)
        shift = min(51, 62 - max(0, int(len(z) - 1).bit_length()))
        f(shift, 0.0 if temperature == 0 else 1.0 / temperature, int(temperature == 0), z.max(), z.ctypes.data, len(z), out.ctypes.data)
        return out
    return run


@pytest.mark.parametrize("vocab,allowed,temperature", [(8192, 102, 1.0), (32000, 100, 0.1), (128256, 40, 0.05), (50021, 100, 0.1), (9000, 500, 0.0), (9000, 20, np.inf), (9000, 20, 1e-30)])
def test_masked_logits_are_in_no_bin(bins, vocab, allowed, temperature):
    """A vector of eight logits has one of a bin's if and only if the bin counts one of them: no more vectors than logits, however many stand beside a mask."""
    rng = np.random.default_rng(vocab)
    z = np.full(vocab, -np.inf, np.float32)
    at = rng.choice(vocab, allowed, replace=False)
    z[at] = rng.standard_normal(allowed) * 20
    b = bins(z, temperature)
    assert (b[np.isneginf(z)] == -1).all() and (b[at] >= 0).all() and (b < 2048).all()
    eights = np.concatenate([b, np.full(-len(b) % 8, -1)]).reshape(-1, 8)
    for one in np.unique(b[at]):
        assert (eights == one).any(axis=1).sum() <= (b[at] == one).sum()


def test_rows_of_8_bits_go_whole_while_registers_hold_them():
    """They are counted, not weighed: nothing for other workgroups to share.  Of 16 bits few long rows go in parts, which need a workspace."""
    from paper_2105_00053_amd import build, generate
    if not os.path.exists(build.LIB):
        build.build()
    need = generate._load().posit_sample_workspace
    for fz in (0, 3, 4):  # posit<8,0>, (8,1), (8,2)
        for rows, vocab in ((1, 16385), (1, 50021), (32, 50021), (1, 131072), (64, 131072), (64, 150001), (128, 300007)):
            assert need(fz, rows, vocab) == 0, (fz, rows, vocab)
        assert need(fz, 1, 131073) > 0 and need(fz, 8, 200003) > 0
    for fz in (1, 102, 100):
        assert need(fz, 1, 16385) > 0 and need(fz, 32, 50021) > 0 and need(fz, 1, 16384) == 0 and need(fz, 128, 50021) == 0


def test_bins_fall_with_the_logits(bins):
    z = np.sort(np.concatenate([np.random.default_rng(1).standard_normal(3000) * 30, [3.4e38, 1e20, -1e20, -3.4e38, 0.0, -0.0]]))[::-1]
    for temperature in (0.0, 1e-30, 0.05, 1.0, 1e30, np.inf):
        for top in (0, 2, 5):  # the largest logits, and rows without them
            b = bins(z[top:], temperature)
            if 0 < temperature < np.inf:
                assert (np.diff(b) >= 0).all() and b[0] == 0 and b.max() <= 2047
            else:  # all in one, but for differences that are infinite
                assert set(b.tolist()) <= {0, 2047} and b[0] == 0
