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


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_non_finite_gradients_stay_visible(layers, bad, dtype):
    """As without pruning: in the row of the input gradient and the row of the weight gradient that they meet."""
    torch.manual_seed(1)
    lin, plain = pair(layers, 64, 48, 0.6)
    for layer in (lin, plain):
        x = torch.randn(40, 64, device="cuda").to(dtype).requires_grad_()
        up = torch.exp(torch.randn(40, 48, device="cuda") - 8).to(dtype)
        up[7, 5] = bad
        layer(x).backward(up)
        assert bool((~torch.isfinite(x.grad[7])).all()) and bool((~torch.isfinite(layer.weight.grad[5])).all())


def test_finite_gradients_are_what_the_library_prunes_them_to(lgn, layers):
    g = torch.exp(2 * torch.randn(300, 100, device="cuda") - 12) * torch.randn(300, 100, device="cuda").sign()
    out, res, ws = torch.empty_like(g), lgn.new_results(1, "cuda"), lgn.new_workspace([g.numel()], "cuda")
    lgn.lgn_compress_layers([lgn.make_layer(g, out, lgn.MODE_PRUNE, S=0.7, seed=9)], res, ws)
    assert torch.equal(layers._pruned(g, 0.7, 9), out)


def test_layers_with_seeds_of_their_own(layers):
    """The same gradient in two layers: different places with different seeds, the same with the same."""
    up = torch.exp(2 * torch.randn(200, 64, device="cuda") - 12)
    zeros = []
    for seed in (1 << 32, 2 << 32, 1 << 32):
        lin = layers.Fp8Linear(64, 64, sparsity=0.5, device="cuda", seed=seed)
        assert lin.seed == seed
        zeros.append(layers._pruned(up, lin.sparsity, lin.seed) == 0)
        lin.advance()
        assert lin.seed == seed + 1
    assert torch.equal(zeros[0], zeros[2]) and int((zeros[0] != zeros[1]).sum()) > 1000
