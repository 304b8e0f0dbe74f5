"""The draw of a token from rows that are mostly masked, as by a grammar: limits that reach the logits far below the largest, in rows held in registers, read again, and cut into parts."""
import numpy as np
import pytest
import torch

import lm_util as lu
import paper_2105_00053_amd as pn
from test_gpu_generate_sample import check, run

pytestmark = pytest.mark.gpu


def masked(rng, rows, vocab, allowed, spread):
    """Logits of -inf but for `allowed` of each row, which lie up to `spread` below its largest."""
    z = np.full((rows, vocab), -np.inf, np.float32)
    for r in range(rows):
        z[r, rng.choice(vocab, allowed, replace=False)] = -spread * rng.random(allowed)
    return z


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(5, 8193), (5, 16001), (18, 16500), (2, 16500), (33, 33001), (3, 131072), (1, 131072)])
@pytest.mark.parametrize("allowed", [20, 140, 500])
def test_top_k_over_a_mask(fmt, rows, vocab, allowed):
    """100 temperatures from the largest down: logits of a weight, of none, and in the last bin some hundreds with thousands of -inf beside them."""
    rng = np.random.default_rng(rows + vocab + allowed)
    z, u = masked(rng, rows, vocab, allowed, 100.0), rng.random(rows).astype(np.float32)
    for k in (allowed // 8, allowed // 2, allowed - 1, allowed, allowed + 5):  # before, inside and behind the last bin's
        check(z, fmt, u, top_k=k)
    check(z * 0.05, fmt, u, top_k=allowed - 3, temperature=0.05)
    check(z, fmt, u, top_k=allowed - 2, top_p=0.9)
    check(z, fmt, u, top_k=allowed // 2 + 3, min_p=0.01)
    check(z, fmt, u, top_k=allowed - 5, top_p=0.99, min_p=1e-7, temperature=0.9)


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(20, 20011), (2, 131072), (70, 66001)])
def test_a_last_bin_of_thousands(fmt, rows, vocab):
    """More logits in the last bin than are listed: they are counted by their bits, beside a mask as without one."""
    rng = np.random.default_rng(vocab)
    z = masked(rng, rows, vocab, 2500, 400.0)
    few = rows if rows < 3 else 3  # of many rows the first are looked at, the others fill the launch
    u = rng.random(rows).astype(np.float32)
    for k in (100, 1200, 2499):
        check(z[:few], fmt, u[:few], top_k=k)
        got = [x[:few] for x in run(z, fmt, u, top_k=k)[0]]
        assert all(np.array_equal(a, b) for a, b in zip(got, run(z[:few], fmt, u[:few], top_k=k)[0]))


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
def test_the_same_every_time(fmt):
    rng = np.random.default_rng(8)
    z, u = masked(rng, 3, 128256, 40, 6.0), rng.random(3).astype(np.float32)
    t, dev = lu.to_format(z, fmt), lambda v, kind: torch.full((3,), v, dtype=kind, device="cuda")
    how = dict(temperature=dev(0.05, torch.float32), top_k=dev(20, torch.int32))
    first = pn.posit_sample(t, torch.from_numpy(u).cuda(), fmt, **how)
    assert first[2].tolist() == [20] * 3
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(first, pn.posit_sample(t, torch.from_numpy(u).cuda(), fmt, **how)))


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(6, 9001), (6, 40003), (6, 700), (2, 70001)])
def test_ends_of_the_temperatures_over_a_mask(fmt, rows, vocab):
    """The likeliest alone, shares alike, all weight on one: bins of no width, one bin for all, and nearly all in the last."""
    rng = np.random.default_rng(rows * vocab)
    for allowed in (1, 40, 650):
        z = masked(rng, rows, vocab, allowed, 30.0)
        z[0, z[0] > -np.inf] = 2.5                                    # equal ones
        z[1, rng.choice(np.flatnonzero(z[1] > -np.inf), 1)] = 3e38    # differences that are infinite, or nearly
        z[1, rng.choice(np.flatnonzero(z[1] > -np.inf), 1)] = -3e38
        u = rng.random(rows).astype(np.float32)
        for temperature in (0.0, np.inf, 1e30, 1e-30, 1e-42):
            check(z, fmt, u, temperature=temperature)
            check(z, fmt, u, temperature=temperature, top_k=allowed // 2 + 1)
            check(z, fmt, u, temperature=temperature, top_k=allowed - allowed // 4, top_p=0.7, min_p=0.2)
