"""What Fp8Linear keeps for its backward pass is autograd's: hooks on saved tensors see it, checkpointing drops and
recomputes it, and it is gone after the pass."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers(lgn):
    from paper_2006_08173_b200 import layers as mod
    return mod


def gradients(lin, x, run):
    x.grad = lin.weight.grad = None
    run().square().sum().backward()
    return x.grad, lin.weight.grad


def test_hooks_and_checkpointing(layers):
    lin = layers.Fp8Linear(96, 48, device="cuda")
    x = torch.randn(37, 96, device="cuda", requires_grad=True)
    want = gradients(lin, x, lambda: lin(x))
    packed = []

    def pack(t):
        packed.append(t)
        return t.cpu()
    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.cuda()):
        got = gradients(lin, x, lambda: lin(x))
    assert sum(t.dtype == torch.uint8 for t in packed) == 2        # the codes of the weights and of the input
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    got = gradients(lin, x, lambda: torch.utils.checkpoint.checkpoint(lin, x, use_reentrant=False))
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_kept_only_until_the_pass(layers):
    lin = layers.Fp8Linear(96, 48, device="cuda")
    x = torch.randn(37, 96, device="cuda", requires_grad=True)
    y = lin(x)
    up = torch.ones_like(y)
    y.backward(up, retain_graph=True)
    once = x.grad.clone()
    y.backward(up)
    assert torch.equal(x.grad, 2 * once)
    with pytest.raises(RuntimeError):
        y.backward(up)
