"""autograd.first_order_only on the CPU, where no kernel is needed to see what a second derivative does."""
import pytest
import torch

from paper_2603_25011_amd.autograd import first_order_only


class Square(torch.autograd.Function):
    """x^2 whose gradient is filled without a graph, as a library fills it."""

    @staticmethod
    def forward(ctx, x, other):
        ctx.save_for_backward(x)
        return x * x

    @staticmethod
    def backward(ctx, dy):
        x, = ctx.saved_tensors
        dx = torch.empty_like(x)
        dx.copy_((2 * x * dy).detach())
        return first_order_only("square", (dx, None), (x, dy))


def test_gradients_pass_and_their_gradients_raise():
    x = torch.tensor([1.0, -3.0], requires_grad=True)
    Square.apply(x, None).sum().backward()
    assert x.grad.tolist() == [2.0, -6.0] and x.grad.grad_fn is None
    g, = torch.autograd.grad(Square.apply(x, None).sum(), x, create_graph=True)
    assert g.tolist() == [2.0, -6.0]
    total = (x ** 2).sum() + g.pow(2).sum()
    with pytest.raises(RuntimeError, match="square"):
        total.backward(retain_graph=True)
    with pytest.raises(RuntimeError, match="square"):
        torch.autograd.grad(total, x)
    dy = torch.ones(2, requires_grad=True)
    g, = torch.autograd.grad(Square.apply(x, None), x, dy, create_graph=True)
    with pytest.raises(RuntimeError, match="square"):
        torch.autograd.grad(g.sum(), dy)
