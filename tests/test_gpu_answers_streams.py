"""Calls on a stream that is not their tensors' own: memory that its own stream has freed is not handed out again before the call has read it."""
import numpy as np
import pytest
import torch

from paper_1907_07346_amd import binding as b
from paper_1907_07346_amd import workloads as wl
from tests.test_gpu_answers import BF16, F32, calls

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("which", range(4))
def test_inputs_freed_while_another_stream_is_busy(which, dtype):
    inputs, f = calls(np.random.default_rng(which), 20, 600, 2000, 128, 20000, dtype)[which]
    want = f(*inputs)
    side = torch.cuda.Stream()
    copies = [t.clone() for t in inputs]
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)                             # the side stream is busy for some 10 ms
    got = f(*copies, stream=side)
    sizes = [(t.shape, t.dtype) for t in copies]
    del copies
    others = [torch.full(shape, 3, dtype=kind, device="cuda") for shape, kind in sizes for _ in range(4)]
    torch.cuda.synchronize()
    for a, w in zip(got, want):
        assert torch.equal(a, w), "the call read memory that belonged to others already"
    assert others


def test_a_handles_message_on_another_stream():
    """The message's memory is the library's own; the call's stream waits for the step's, as it has to."""
    n, V, D = 4, 40, 128
    cfg, keep = b.make_config(n, V * D, wl.TOPO_RING, wl.KIND_QUANT_MAXABS, 0.05, 0.3, bits=4, block=64, seed=1)
    ds = b.DeepSqueeze(cfg, keep)
    ds.ds_step(torch.randn((n, V * D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)))
    x = torch.randn((3, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    want, back = ds.ds_product(1, x, V), ds.ds_product_gradient(1, x[:, :V].contiguous(), D)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, got_back = ds.ds_product(1, x, V, stream=side), ds.ds_product_gradient(1, x[:, :V].contiguous(), D, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(got_back, back)
    ds.ds_destroy()
