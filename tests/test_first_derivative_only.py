"""The wrapper around backward passes that fill their gradients outside autograd, on the CPU."""
import pytest
import torch

from paper_2609_14306_b200.autograd import first_derivative_only


class Square(torch.autograd.Function):
    """x^2, whose gradient leaves autograd on its way."""

    @staticmethod
    def forward(ctx, x, _unused):
        ctx.save_for_backward(x)
        return x * x

    @staticmethod
    @first_derivative_only
    def backward(ctx, g):
        (x,) = ctx.saved_tensors
        return torch.from_numpy(2 * (x * g).detach().numpy()), None


def test_first_derivatives_are_unchanged():
    x = torch.tensor([1.0, -2.0], requires_grad=True)
    Square.apply(x, None).sum().backward()
    assert torch.equal(x.grad, torch.tensor([2.0, -4.0])) and not x.grad.requires_grad
    (g,) = torch.autograd.grad(Square.apply(x, None).sum(), x, create_graph=True)
    assert torch.equal(g.detach(), torch.tensor([2.0, -4.0]))


@pytest.mark.parametrize("upstream_needs_grad", [False, True])
def test_second_derivatives_raise(upstream_needs_grad):
    x = torch.tensor([1.0, -2.0], requires_grad=True)
    y = Square.apply(x, None)
    loss = (y * y if upstream_needs_grad else y).sum()
    (g,) = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        (g.square().sum() + loss).backward()
