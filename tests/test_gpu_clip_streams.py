"""Gradients of one stream, laid and clipped on another: memory that its own stream has freed is not handed out before the call is done with it."""
import pytest
import torch

from paper_1907_07346_amd import binding as b

pytestmark = pytest.mark.gpu
N = 1 << 20


@pytest.mark.parametrize("at_once", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_tensors_of_another_stream_than_the_tables(in_place, at_once):
    side = torch.cuda.Stream()
    for _ in range(5):
        x = [torch.ones(N, device="cuda") for _ in range(4)]
        out = torch.zeros((1, 4 * N), device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g = x if at_once else b.Gradients(x)
            if not at_once:                           # (laying waits for its stream)
                torch.cuda._sleep(20_000_000)         # the side stream is busy for some 10 ms
            norm = b.ds_clip(g, 1.0, out=None if in_place else out, stream=side)
        del x, g
        others = [torch.full((N,), 9.0, device="cuda") for _ in range(8)]         # on the current stream: may take the freed tensors' places
        torch.cuda.synchronize()
        assert float(norm) == 2048.0
        assert in_place or bool((out == 1.0 / 2048).all()), "the call read memory that belonged to others already"
        assert all(bool((t == 9.0).all()) for t in others), "the call wrote to memory that belonged to others already"
        del others


def test_gradients_that_a_graph_has_saved():
    """A second derivative whose first was clipped in place: refused, not wrong."""
    x = torch.randn(5000, device="cuda", requires_grad=True)
    grad, = torch.autograd.grad((x ** 3).sum(), x, create_graph=True)
    again = (grad * grad).sum()                       # saves grad
    with torch.no_grad():
        b.ds_gradient_norm([grad])
        torch.autograd.grad(again, x, retain_graph=True)
        b.ds_clip([grad], 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(again, x)
