"""By which numbers ds_sample divides its work, as far as its scratch memory and what the binding hands on tell: host code alone."""
import ctypes

import numpy as np
import pytest
import torch

from paper_1907_07346_amd import binding as b


def work(**kw):
    args = dict(rows=1, vocab=131072, dtype=0, top_k=0, temperature=1.0, top_p=0.9, min_p=0.0, reserved=0)
    args.update(kw)
    return b.lib().ds_sample_work_bytes(ctypes.byref(b.ds_sampling(**args)))


@pytest.mark.parametrize("dtype,vocab", [(0, 131072), (2, 131072), (0, 8 << 20), (1, 1 << 20)])
def test_the_largest_alone_is_not_split(dtype, vocab):
    """At temperature 0 one logit is kept, as with top_k = 1."""
    assert work(dtype=dtype, vocab=vocab) > 0
    assert work(dtype=dtype, vocab=vocab, top_k=1) == 0
    assert work(dtype=dtype, vocab=vocab, temperature=0.0) == 0
