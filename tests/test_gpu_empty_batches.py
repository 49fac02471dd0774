"""The modules on batches without a row: gradients of zeros, whatever strides the incoming gradient has."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers(lgn):
    from paper_2006_08173_b200 import layers as mod
    return mod


@pytest.mark.parametrize("sparsity", [0.0, 0.5])
@pytest.mark.parametrize("how", ["expanded", "plain"])
def test_linear(layers, how, sparsity):
    lin = layers.Fp8Linear(64, 32, sparsity, device="cuda")
    x = torch.zeros(0, 64, device="cuda", requires_grad=True)
    y = lin(x)
    assert y.shape == (0, 32)
    if how == "expanded":
        y.sum().backward()
    else:
        y.backward(torch.zeros(0, 32, device="cuda"))
    assert x.grad.shape == (0, 64) and bool((lin.weight.grad == 0).all())


def test_embedding(layers):
    emb = layers.Embedding(50, 40, device="cuda")
    out = emb(torch.zeros(2, 0, dtype=torch.int64, device="cuda"))
    assert out.shape == (2, 0, 40)
    out.sum().backward()
    assert bool((emb.weight.grad == 0).all())


def test_matrices_without_elements(lgn):
    none = torch.zeros(1, device="cuda").expand(0, 5), torch.zeros(1, device="cuda").expand(5, 0)
    for x in none:
        q, t = lgn.lgn_fp8_quantize(x, transposed=True)
        assert (q.rows, q.k, t.rows, t.k) == (*x.shape, *x.shape[::-1])
