"""The differentiable functions have first derivatives only: a second one is refused, not left out of the result."""
import pytest
import torch

import paper_2609_14306_b200 as vp

pytestmark = pytest.mark.gpu


def penalised(loss, *inputs):
    """A loss with a penalty on its own gradient, back-propagated."""
    grads = torch.autograd.grad(loss, inputs, create_graph=True)
    (sum(g.float().square().sum() for g in grads) + loss).backward()


def layer_norm():
    x, w, b = (torch.randn(*s, device="cuda", requires_grad=True) for s in ((6, 40), (40,), (40,)))
    return vp.layer_norm(x, w, b).square().sum(), (x, w, b)


def policy_loss():
    x = torch.randn(60, device="cuda", requires_grad=True)
    off = torch.tensor([0, 25, 60], device="cuda")
    return vp.policy_loss(x, x.detach() + 0.1, torch.randn(2, device="cuda"), off, ref_logp=x.detach() - 0.1, kl_coef=0.1)[0], (x,)


def preference_loss():
    x = torch.randn(60, device="cuda", requires_grad=True)
    return vp.preference_loss(x, torch.tensor([0, 25, 60], device="cuda"))[0], (x,)


def head(mean=False):
    H = (0.2 * torch.randn(128, 64, device="cuda")).bfloat16().requires_grad_(True)
    W = (0.2 * torch.randn(512, 64, device="cuda")).bfloat16().requires_grad_(True)
    labels = torch.randint(0, 512, (128,), device="cuda")
    if mean:
        return vp.vocab_proj_cross_entropy_mean(H, W, labels, block_v=256), (H, W)
    return vp.vocab_proj_cross_entropy(H, W, labels, block_v=256).sum(), (H, W)


def head_mean():
    return head(mean=True)


@pytest.mark.parametrize("case", [layer_norm, policy_loss, preference_loss, head, head_mean])
def test_second_derivatives_are_refused(case):
    torch.manual_seed(0)
    loss, inputs = case()
    with pytest.raises(RuntimeError, match="second derivative"):
        penalised(loss, *inputs)
    # a graph of the gradient alone, not differentiated, changes nothing
    torch.manual_seed(0)
    loss, inputs = case()
    plain = torch.autograd.grad(loss, inputs, retain_graph=True)
    graphed = torch.autograd.grad(loss, inputs, create_graph=True)
    assert all(torch.equal(p, q.detach()) for p, q in zip(plain, graphed))
