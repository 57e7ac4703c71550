"""Tokens drawn from short rows, a wave each: up to 512 logits, and up to 2048 where there are many rows of fp32 or fp16, against a sorted list in 64 bits.  Tolerances as
in test_gpu_sample.py."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sample import BF16, F16, F32, check, uniform

pytestmark = pytest.mark.gpu

ALIKE = [dict(), dict(top_p=0.9), dict(top_p=0.45), dict(top_k=40), dict(top_k=77, top_p=0.6), dict(min_p=0.3), dict(min_p=0.5), dict(top_k=100, min_p=0.2, top_p=0.97),
         dict(temperature=3.0), dict(temperature=0.02, top_p=0.999), dict(temperature=0.0)]


def alike(vocab, dtype, seed):
    """Rows with more logits than a wave has lanes whose distances to the largest are one number in 64 bits, though they differ."""
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((9, vocab))
    z[0] *= 1e-20                                                                 # behind one of 1
    z[0, vocab // 3] = 1.0
    z[1] = -np.abs(z[1]) * 1e-30
    z[1, 0] = z[1, vocab - 1] = 0.25
    z[2] = np.where(rng.random(vocab) < 0.5, z[2], 1e-25 * z[2])                   # among ordinary ones
    z[3] = rng.integers(-1000, 1000, vocab) * 2.0 ** (-149 if dtype == F32 else -133)
    z[3, vocab // 2] = 3.0
    z[4] = np.where(rng.random(vocab) < 0.3, np.where(rng.random(vocab) < 0.5, 0.0, -0.0), 1e-20 * z[4])
    z[4, 1] = 2.0
    z[5] *= 1e-20                                                                 # nothing in front: no two are alike that are not equal
    z[6] = 1e-22 * z[6]
    z[6, ::3] = -np.inf
    z[6, 1] = 0.5
    z[7] = 1e-20 * np.round(z[7])
    z[7, 2] = 1.5
    z[8] = 1e-18 * z[8] + np.where(rng.random(vocab) < 0.1, 1.0, 0.0)
    return torch.from_numpy(z).to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [65, 66, 130, 300, 511, 512])
def test_logits_that_are_alike_but_not_equal(vocab, dtype):
    z = alike(vocab, dtype, seed=vocab)
    for i, f in enumerate(ALIKE):
        check(z, uniform(len(z), 100 * vocab + i), **f)


def test_logits_that_are_alike_in_many_rows():
    z = alike(2048, F32, seed=1).repeat(228, 1)[:2050]
    z[50:] = torch.roll(z[50:], 5, dims=1)
    for i, f in enumerate((dict(), dict(top_p=0.9), dict(min_p=0.3, temperature=0.9))):
        check(z, uniform(len(z), i), **f)
