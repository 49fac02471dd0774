"""The modules on transposed, broadcast and sliced matrices: the bits of the same call on contiguous copies."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers(lgn):
    from paper_2006_08173_b200 import layers as mod
    return mod


def views(rows, cols, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return {"transposed": r(cols, rows).t(), "one row": r(1, cols).expand(rows, cols), "one column": r(rows, 1).expand(rows, cols),
            "every second": r(2 * rows, 2 * cols)[::2, ::2], "part": r(rows, cols + 9)[:, 4:4 + cols], "contiguous": r(rows, cols)}


KINDS = ["transposed", "one row", "one column", "every second", "part", "contiguous"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [1, 37])
def test_linear_input(layers, kind, rows):
    lin = layers.Fp8Linear(96, 48, device="cuda")
    x = views(rows, 96, 1)[kind].requires_grad_()
    same = x.detach().clone(memory_format=torch.contiguous_format).requires_grad_()
    y = lin(x)
    up = torch.randn(rows, 48, device="cuda")
    y.backward(up)
    dw, lin.weight.grad = lin.weight.grad, None
    z = lin(same)
    z.backward(up)
    assert torch.equal(y, z) and torch.equal(x.grad, same.grad) and torch.equal(dw, lin.weight.grad)


@pytest.mark.parametrize("kind", KINDS)
def test_weights_and_gradients(layers, kind):
    up, x = views(37, 48, 2)[kind], torch.randn(37, 96, device="cuda", requires_grad=True)
    got = []
    for copy in (False, True):
        lin, emb = layers.Fp8Linear(96, 48, device="cuda"), layers.Embedding(48, 96, out_dtype=torch.float32, device="cuda")
        for m in (lin, emb):
            w = views(48, 96, 3)[kind]
            m.weight = torch.nn.Parameter(w.clone(memory_format=torch.contiguous_format) if copy else w)
        x.grad = None
        y = lin(x)
        y.backward(up.clone(memory_format=torch.contiguous_format) if copy else up)
        ids = torch.arange(40, device="cuda")
        e = emb(ids)
        e.backward(views(40, 96, 4)[kind])
        got.append([y, x.grad, lin.weight.grad, e, emb.weight.grad])
    assert all(torch.equal(a, b) for a, b in zip(*got))
