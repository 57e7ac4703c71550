"""Whose memory waits for a call on which stream: what Gradients records its table and tensors with.  No GPU: streams and tensors are stand-ins."""
import types

import pytest
import torch

from paper_1907_07346_amd import binding as b


class Held:
    """A tensor that notes the streams it is recorded with."""

    def __init__(self):
        self.streams = []

    def record_stream(self, stream):
        self.streams.append(stream.cuda_stream)


def stream(pointer):
    return types.SimpleNamespace(cuda_stream=pointer, device_index=0)


@pytest.fixture
def laid(monkeypatch):
    """Gradients that were laid on stream 7, and the calls on them with the stream that is current."""
    g = b.Gradients.__new__(b.Gradients)
    g.workers, g.columns, g._g, g._work, g._apart, g._made_on, g._lent_to = 1, 4, b.ds_gradients(), (0, 0), True, 7, set()
    g.table, g.tensors = Held(), [Held(), Held()]
    monkeypatch.setattr(b, "_on_device", lambda *a: 0)
    monkeypatch.setattr(torch.autograd.graph, "increment_version", lambda tensors: None)      # (stand-ins have none)
    monkeypatch.setattr(b, "_new", lambda stream, shape, dtype, like: torch.zeros(shape, dtype=dtype))
    monkeypatch.setattr(b, "lib", lambda: types.SimpleNamespace(ds_gradient_norm=lambda *a: b.DS_OK, ds_clip=lambda *a: b.DS_OK))

    def call(which, current, given=None):
        monkeypatch.setattr(b, "_raw_stream", lambda device: current)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: stream(current))
        b.ds_gradient_norm(g, stream=given) if which == "norm" else b.ds_clip(g, 1.0, stream=given)

    return g, call


@pytest.mark.parametrize("which", ["norm", "clip"])
def test_a_given_stream_is_recorded_though_the_table_was_laid_on_it(laid, which):
    g, call = laid
    call(which, 7, stream(7))                         # the tensors may be of any other
    assert all(set(t.streams) == {7} for t in g.tensors)


@pytest.mark.parametrize("which", ["norm", "clip"])
def test_other_streams_are_recorded_and_the_tables_own_is_not(laid, which):
    g, call = laid
    call(which, 7)
    assert all(t.streams == [] for t in (g.table, *g.tensors))
    call(which, 9)
    call(which, 7, stream(11))
    call(which, 9)
    assert all(set(t.streams) == {9, 11} for t in (g.table, *g.tensors))
