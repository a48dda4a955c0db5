"""Layer norm where shapes, widths and sizes change the path that runs.  Oracle, bounds and helpers are those of
test_gpu_layer_norm."""
import pytest
import torch

import paper_2609_14306_b200 as vp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(48,), (1, 48), (1, 1, 48)])
def test_gradients_have_their_parameters_shapes(shape):
    """weight and bias of d elements in any shape: what the parameters have, their gradients have."""
    torch.manual_seed(1)
    x = torch.randn(9, 48, device="cuda", requires_grad=True)
    w, b = (torch.randn(shape, device="cuda", requires_grad=True) for _ in range(2))
    up = torch.randn(9, 48, device="cuda")
    (vp.layer_norm(x, w, b) * up).sum().backward()
    flat_w, flat_b = (t.detach().reshape(48).clone().requires_grad_(True) for t in (w, b))
    (vp.layer_norm(x.detach(), flat_w, flat_b) * up).sum().backward()
    assert w.grad.shape == shape and b.grad.shape == shape
    assert torch.equal(w.grad.reshape(48), flat_w.grad) and torch.equal(b.grad.reshape(48), flat_b.grad)
