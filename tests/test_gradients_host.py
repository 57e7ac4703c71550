"""What the calls on gradients in many tensors refuse, and their sizes: host code alone, no kernel is launched."""
import ctypes

import numpy as np
import pytest
import torch

from paper_1907_07346_amd import binding as b

BIG = 1 << 40                                       # an address that is never touched


def tensors(*of):
    """(data, count, dtype, worker) each."""
    return (b.ds_tensor * max(len(of), 1))(*[b.ds_tensor(*t) for t in of])


def lay(of, workers=2, table=BIG, size=1 << 40, count=None, out=True, null=False):
    buf, g = ctypes.create_string_buffer(256), b.ds_gradients()
    st = b.lib().ds_gradients_lay(None if null else tensors(*of), len(of) if count is None else count, workers, table, size,
                                  ctypes.byref(g) if out else None, None, buf, 256)
    return st, buf.value.decode()


GOOD = [(BIG, 100, 0, 0), (2 * BIG, 16385, 1, 1)]


@pytest.mark.parametrize("of,call,needle", [
    (GOOD, dict(workers=0), "workers"), (GOOD, dict(workers=1 << 20), "workers"), (GOOD, dict(workers=1), "workers"), (GOOD, dict(null=True), "NULL"),
    (GOOD, dict(count=1 << 24), "2^24"), ([(BIG, 1, 0, 1), (BIG, 1, 0, 0)], {}, "descend"), ([(BIG, 1, 0, -1)], {}, "workers"),
    ([(BIG, 1, 3, 0)], {}, "dtype"), ([(BIG, 1, -1, 0)], {}, "dtype"), ([(BIG, 1 << 40, 0, 0)], {}, "2^40"), ([(None, 1, 0, 0)], {}, "NULL"),
    ([(BIG, (1 << 40) - 1, 0, 0), (BIG, 1, 0, 0)], {}, "2^40"), ([(BIG + 2, 1, 0, 0)], {}, "aligned"), ([(BIG + 1, 1, 2, 0)], {}, "aligned"),
    ([((1 << 64) - 4, 2, 0, 0)], {}, "address space"), (GOOD, dict(table=None), "table_dev"), (GOOD, dict(size=100), "table_dev"),
    (GOOD, dict(table=BIG + 8), "16-byte"), (GOOD, dict(out=False), "out is NULL"),
])
def test_lists_that_are_refused(of, call, needle):
    st, why = lay(of, **call)
    assert st == b.DS_EINVAL and needle in why, why


def test_too_many_tiles_are_refused():
    of = [(BIG, (1 << 40) - 1, 1, w) for w in range(64)]
    assert lay(of, workers=64)[0] == b.DS_EINVAL and b.lib().ds_gradients_bytes(tensors(*of), len(of), 64) == 0


def test_bytes_of_a_table():
    L = b.lib()
    record = 48
    assert L.ds_gradients_bytes(tensors(*GOOD), 2, 2) == 3 * record + 3 * 8 + 3 * 4
    assert L.ds_gradients_bytes(tensors(*GOOD), 2, 7) == 3 * record + 8 * 8 + 3 * 4
    assert L.ds_gradients_bytes(None, 0, 1) == record + 2 * 8
    assert L.ds_gradients_bytes(tensors((None, 0, 2, 0)), 1, 1) == 2 * record + 2 * 8
    assert L.ds_gradients_bytes(tensors(*GOOD), 2, 1) == 0


def description(**kw):
    args = dict(table_dev=BIG, workers=2, tensors=2, tiles=3, columns=16385, worker_tiles=2)
    args.update(kw)
    args.setdefault("table_bytes", (args["tensors"] + 1) * 48 + (args["workers"] + 1) * 8 + args["tiles"] * 4)
    return b.ds_gradients(**args)


def clip(g, max_norm=1.0, out=2 * BIG, ld=16385, norm=3 * BIG, work=4 * BIG, size=1 << 40):
    buf = ctypes.create_string_buffer(256)
    st = b.lib().ds_clip(ctypes.byref(g) if g else None, max_norm, out, ld, norm, work, size, None, buf, 256)
    return st, buf.value.decode()


@pytest.mark.parametrize("kw,call,needle", [
    (None, {}, "NULL"), (dict(table_dev=None), {}, "lay"), (dict(table_dev=BIG + 8), {}, "lay"), (dict(workers=0), {}, "lay"),
    (dict(table_bytes=17), {}, "lay"), (dict(worker_tiles=4), {}, "lay"), ({}, dict(max_norm=-1.0), "max_norm"),
    ({}, dict(max_norm=float("nan")), "max_norm"), ({}, dict(out=2 * BIG + 2), "4-byte"), ({}, dict(norm=3 * BIG + 1), "4-byte"),
    ({}, dict(ld=16384), "g_ld"), ({}, dict(ld=1 << 63), "address space"), ({}, dict(out=BIG), "table"), ({}, dict(work=None), "work_dev"),
    ({}, dict(size=(3 + 2) * 8 - 1), "work_dev"), ({}, dict(work=4 * BIG + 8), "16-byte"),
])
def test_clip_refuses(kw, call, needle):
    st, why = clip(description(**kw) if kw is not None else None, **call)
    assert st == b.DS_EINVAL and needle in why, why


@pytest.mark.parametrize("norm,work,size,needle", [(None, BIG, 1 << 30, "NULL"), (BIG + 2, BIG, 1 << 30, "4-byte"), (BIG, None, 0, "work_dev"), (BIG, BIG, 23, "work_dev")])
def test_norm_refuses(norm, work, size, needle):
    buf = ctypes.create_string_buffer(256)
    assert b.lib().ds_gradient_norm(ctypes.byref(description()), norm, work, size, None, buf, 256) == b.DS_EINVAL
    assert needle in buf.value.decode()


def test_scratch_bytes():
    L = b.lib()
    assert L.ds_gradient_norm_work_bytes(ctypes.byref(description())) == 3 * 8
    assert L.ds_clip_work_bytes(ctypes.byref(description())) == (3 + 2) * 8
    assert L.ds_clip_work_bytes(ctypes.byref(description(workers=0))) == 0 and L.ds_gradient_norm_work_bytes(None) == 0


# ---- the binding, before it asks the library --------------------------------------------------------

def refused(call, needle):
    with pytest.raises(b.DsqError, match=needle) as e:
        call()
    assert e.value.status == b.DS_EINVAL


def test_tensors_that_are_refused(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for t in (torch.zeros(4, dtype=torch.float64), torch.zeros((4, 6))[:, ::2], torch.zeros((4, 6)).t(), None):
        refused(lambda: b.Gradients([[t]]), "contiguous")
        refused(lambda: b.ds_gradient_norm([[torch.zeros(3), t]]), "contiguous")
    leaf = torch.zeros(4, requires_grad=True)
    refused(lambda: b.Gradients([leaf]), "requires a gradient")
    with torch.no_grad():
        refused(lambda: b.Gradients([leaf]), "current CUDA device")
    refused(lambda: b.Gradients([torch.zeros(4)]), "current CUDA device")


def laid(sizes, at, pitch=None):
    """A Gradients of one fp32 tensor per worker at the given addresses, whose table is never used."""
    g = b.Gradients.__new__(b.Gradients)
    g.workers, g.device, g.columns = len(sizes), 0, max(sizes)
    g._lo = np.array(at, np.uint64)
    g._hi = g._lo + np.uint64(4) * np.array(sizes, np.uint64)
    g._f32, g._worker = np.ones(len(sizes), bool), np.arange(len(sizes), dtype=np.uint64)
    g._column = np.zeros(len(sizes), np.uint64)
    g._span = (min(at), int(g._hi.max()))
    return g


def test_results_over_gradients():
    out = torch.zeros((2, 12))
    at = out.data_ptr()
    assert not laid([10, 10], [at, at + 48])._overlapped(at, 12)                  # where they go
    assert laid([10, 10], [at, at + 40])._overlapped(at, 12)
    assert laid([10, 10], [at + 4, BIG])._overlapped(at, 12)
    assert not laid([10, 10], [at - 40, at + 4 * 22])._overlapped(at, 12)         # before it, and behind the last row's elements
    assert laid([10, 10], [at - 36, BIG])._overlapped(at, 12)
    assert laid([10, 10], [at + 48, at])._overlapped(at, 12)                      # the wrong rows
