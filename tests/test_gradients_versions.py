"""ds_clip changes tensors behind torch's back: their version counters say so, as after any operation in place.  No GPU: the library is a stand-in."""
import types

import pytest
import torch

from paper_1907_07346_amd import binding as b


@pytest.fixture
def clip(monkeypatch):
    def done(status):
        monkeypatch.setattr(b, "lib", lambda: types.SimpleNamespace(ds_clip=lambda *a: status, ds_gradient_norm=lambda *a: status))

    monkeypatch.setattr(b, "_on_device", lambda *a: 0)
    monkeypatch.setattr(b, "_raw_stream", lambda device: 7)
    done(b.DS_OK)

    def laid(tensors):
        g = b.Gradients.__new__(b.Gradients)
        g.workers, g.columns, g._g, g._work, g._apart, g._made_on, g._lent_to = 1, sum(t.numel() for t in tensors), b.ds_gradients(), (0, 0), True, 7, set()
        g.table, g.tensors, g._span = torch.zeros(16, dtype=torch.uint8), [t.detach() for t in tensors], (0, 0)
        return g

    laid.done = done
    return laid


def test_what_is_scaled_in_place(clip):
    x = [torch.ones(3), torch.ones(4)]
    g = clip(x)
    before = [t._version for t in x]
    b.ds_gradient_norm(g)
    assert [t._version for t in x] == before
    b.ds_clip(g, 1.0)
    assert all(t._version > v for t, v in zip(x, before))


def test_a_result_in_rows(clip):
    x, out = [torch.ones(3)], torch.zeros((1, 3))
    versions = x[0]._version, out._version
    b.ds_clip(clip(x), 1.0, out=out)
    assert x[0]._version == versions[0] and out._version > versions[1]


def test_a_gradient_that_a_graph_has_saved(clip):
    leaf, x = torch.ones(3, requires_grad=True), torch.ones(3)
    y = (leaf * x).sum()                              # saves x
    with torch.no_grad():
        b.ds_clip(clip([x]), 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_tensors_without_versions(clip):
    with torch.inference_mode():
        x, out = [torch.ones(3)], torch.zeros((1, 3))
    b.ds_clip(clip(x), 1.0)
    b.ds_clip(clip(x), 1.0, out=out)
    with torch.inference_mode():
        b.ds_clip(clip(x), 1.0)


def test_calls_that_are_refused_change_nothing(clip):
    x, out = [torch.ones(3)], torch.zeros((1, 3))
    g, versions = clip(x), (x[0]._version, out._version)
    clip.done(b.DS_EINVAL)
    for where in (None, out):
        with pytest.raises(b.DsqError):
            b.ds_clip(g, -1.0, out=where)
    assert (x[0]._version, out._version) == versions
