"""Fp8Linear with its neural gradient pruned, on the gradients that autograd hands over."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers(lgn):
    from paper_2006_08173_b200 import layers as mod
    return mod


def pair(layers, k, n, sparsity):
    """A pruning layer and one without pruning on the same weights."""
    a, b = layers.Fp8Linear(k, n, sparsity=sparsity, device="cuda"), layers.Fp8Linear(k, n, device="cuda")
    b.weight.data.copy_(a.weight.data)
    return a, b


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 3, 7, 8])
def test_a_slice_of_a_larger_gradient(layers, rows, dtype):
    """The gradient of the second of two concatenated outputs starts `rows` rows into a buffer: at any element's address."""
    torch.manual_seed(rows)
    lin, plain = pair(layers, 64, 75, 0.5)
    x, other = torch.randn(40, 64, device="cuda").to(dtype), torch.randn(rows, 75, device="cuda").to(dtype)
    other.requires_grad_()
    up = torch.exp(2 * torch.randn(rows + 40, 75, device="cuda") - 12).to(dtype)
    torch.cat([other, lin(x)]).backward(up)
    plain(x).backward(layers._pruned(up[rows:].clone(), 0.5, 0))
    assert torch.equal(lin.weight.grad, plain.weight.grad)
