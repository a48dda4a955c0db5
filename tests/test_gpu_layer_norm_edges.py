"""Layer norm where shapes, widths and sizes change the path that runs.  Oracle, bounds and helpers are those of
test_gpu_layer_norm."""
import pytest
import torch

import paper_2609_14306_b200 as vp
import test_gpu_layer_norm as ln

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


# fp32 rows leave the row kernels where two rows and the weights no longer fit shared memory: above 14336 columns forward and 11320
# backward; 16-bit rows above 16384 columns; aligned rows of up to 512 bytes have kernels of their own.
@pytest.mark.parametrize("dtype,d", [(torch.float32, d) for d in (11316, 11319, 11320, 11321, 11324, 14332, 14336, 14337, 14340, 16384, 16385)]
                         + [(torch.bfloat16, d) for d in (16376, 16383, 16384, 16385, 16392)]
                         + [(torch.float16, d) for d in (255, 256, 257, 264)] + [(torch.float32, d) for d in (127, 128, 129, 132)])
@pytest.mark.parametrize("rows", [1, 5, 300])
def test_both_sides_of_the_switches_between_the_kernels(rows, d, dtype):
    ln.check(*ln.make(rows, d, dtype, torch.float32, seed=d + rows))
