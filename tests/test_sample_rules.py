"""By which numbers ds_sample divides its work, as far as its scratch memory and what the binding hands on tell: host code alone."""
import ctypes
import types

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


def test_a_top_p_of_rows_is_told_to_the_rule(monkeypatch):
    """min_p beside a vector of top_p is not min_p alone: masses of all logits have to be made."""
    asked = []

    def note(s, *args):
        s = s._obj
        asked.append((s.top_k, s.temperature, s.top_p, s.min_p))
        return 0

    monkeypatch.setattr(b, "lib", lambda: types.SimpleNamespace(ds_sample_work_bytes=note, ds_sample=lambda s, *args: b.DS_OK))
    monkeypatch.setattr(b, "_on_device", lambda *a: 0)
    monkeypatch.setattr(b, "_raw_stream", lambda device: 0)
    z, u, each = torch.zeros((3, 10)), torch.zeros(3), torch.full((3,), 0.5)
    b.ds_sample(z, u, min_p=0.05, top_p=each)
    b.ds_sample(z, u, min_p=0.05)
    b.ds_sample(z, u, min_p=0.05, top_p=0.75)
    b.ds_sample(z, u, temperature=each, top_k=each.to(torch.int32), min_p=each)
    assert asked[0][2] < 1.0 and asked[0][3] == np.float32(0.05)
    assert asked[1][2] == 1.0 and asked[2][2] == 0.75
    assert asked[3] == (1, 1.0, 1.0, 0.0)


def test_min_p_alone_is_another_rule():
    assert work(min_p=0.05) > 0 and work(min_p=0.05, top_p=1.0) == 0 and work(top_p=1.0) > 0
