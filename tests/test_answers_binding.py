"""What the binding of the operators on messages refuses before it asks the library: no GPU, no handle."""
import types

import pytest
import torch

from paper_1907_07346_amd import binding as b
from paper_1907_07346_amd import workloads as wl


def handle(algo=wl.ALGO_DEEPSQUEEZE, stepped=True, **kw):
    """A DeepSqueeze whose handle is never used."""
    ds = b.DeepSqueeze.__new__(b.DeepSqueeze)
    ds.cfg, ds._keep = b.make_config(4, 640, wl.TOPO_RING, wl.KIND_QUANT_MAXABS, 0.1, 0.5, bits=4, block=64, algo=algo, **kw)
    ds._h, ds.n, ds.N, ds._stepped = None, 4, 640, stepped
    return ds


@pytest.mark.parametrize("algo", [wl.ALGO_DCD_PSGD, wl.ALGO_CHOCO_SGD])
def test_messages_that_are_differences_are_no_matrix(algo):
    ds = handle(algo)
    for call in (lambda: ds.ds_product(0, torch.zeros((1, 64)), 2), lambda: ds.ds_product_gradient(0, torch.zeros((1, 2)), 64)):
        with pytest.raises(b.DsqError, match="differences") as e:
            call()
        assert e.value.status == b.DS_EINVAL


def test_a_first_step_that_fails_leaves_no_message(monkeypatch):
    ds, answers = handle(stepped=False), iter([b.DS_EHIP, b.DS_EINVAL, b.DS_OK, b.DS_EHIP])
    monkeypatch.setattr(b, "lib", lambda: types.SimpleNamespace(ds_step=lambda *a: next(answers)))
    for status, there in ((b.DS_EHIP, False), (b.DS_EINVAL, False), (b.DS_OK, True), (b.DS_EHIP, True)):
        assert ds.ds_step_raw(0, 640) == status and ds._stepped is there
        if not there:
            with pytest.raises(b.DsqError) as e:
                ds.ds_product(0, torch.zeros((1, 64)), 2)
            assert e.value.status == b.DS_ESTATE


def test_products_that_would_drop_a_gradient_are_refused(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    msg, leaf = torch.zeros(2 * 36, dtype=torch.uint8), torch.zeros((3, 64), requires_grad=True)
    for x in (leaf, leaf * 2):
        for call in (lambda: b.ds_product(msg, x, 2, 64), lambda: b.ds_product_gradient(msg, x[:, :2], 64, 64)):
            with pytest.raises(b.DsqError, match="graph") as e:
                call()
            assert e.value.status == b.DS_EINVAL
            with torch.no_grad(), pytest.raises(b.DsqError, match="current CUDA device"):     # (it goes on to the next check)
                call()
    with pytest.raises(b.DsqError, match="current CUDA device"):
        b.ds_product(msg, leaf.detach(), 2, 64)
