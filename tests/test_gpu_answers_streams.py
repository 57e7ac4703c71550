"""Calls on a stream that is not their tensors' own: memory that its own stream has freed is not handed out again before the call has read it."""
import numpy as np
import pytest
import torch

from paper_1907_07346_amd import binding as b
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
