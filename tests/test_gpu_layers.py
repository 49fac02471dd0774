"""The operators as torch modules, and the example that runs them together."""
import os
import sys

import numpy as np
import pytest
import torch

from fp8_helpers import quantise, to_np

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def layers(lgn):
    from paper_2006_08173_b200 import layers as mod
    return mod


def close(got, want, mag, k, dtype):
    """As for the product itself: groups of 32 added in fp32, one rounding."""
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    tol = ((k + 31) // 32 + 32) * 2.0 ** -23 * mag
    tol = tol + half * (np.abs(want) + tol)
    assert np.all(np.abs(to_np(got) - want) <= tol)


@pytest.mark.parametrize("t,k,n", [(1, 64, 40), (37, 300, 129), (200, 256, 512)])
def test_linear_gradients_follow_the_formulas(layers, t, k, n):
    g = torch.Generator().manual_seed(t)
    lin = layers.Fp8Linear(k, n, device="cuda")
    x = torch.randn(t, k, generator=g).bfloat16().cuda().requires_grad_()
    dy = (1e-4 * torch.randn(t, n, generator=g)).bfloat16().cuda()
    y = lin(x)
    y.backward(dy)
    xv, wv = quantise(to_np(x), 0)[0], quantise(to_np(lin.weight), 0, True)[0]
    close(y, xv @ wv.T, np.abs(xv) @ np.abs(wv).T, k, torch.bfloat16)
    dv = quantise(to_np(dy), 1)[0]
    close(x.grad, dv @ wv, np.abs(dv) @ np.abs(wv), n, torch.bfloat16)
    dt, xt = quantise(to_np(dy).T, 1)[0], quantise(to_np(x).T, 0)[0]
    close(lin.weight.grad, dt @ xt.T, np.abs(dt) @ np.abs(xt).T, t, torch.float32)


def test_linear_takes_broadcast_gradients_and_leading_dimensions(layers):
    lin = layers.Fp8Linear(64, 32, device="cuda")
    x = torch.randn(2, 5, 64, device="cuda").bfloat16().requires_grad_()
    y = lin(x)
    assert y.shape == (2, 5, 32)
    y.sum().backward()                                            # every row's gradient is the same expanded scalar
    assert x.grad.shape == x.shape and bool((x.grad == x.grad[0, 0]).all())


def test_pruned_linear_gradient_is_that_of_the_pruned_input(layers, lgn):
    torch.manual_seed(0)
    lin = layers.Fp8Linear(128, 256, sparsity=0.7, device="cuda")
    plain = layers.Fp8Linear(128, 256, device="cuda")
    plain.weight.data.copy_(lin.weight.data)
    x = torch.randn(512, 128, device="cuda").bfloat16()
    dy = torch.exp(2 * torch.randn(512, 256, device="cuda") - 12).bfloat16()
    lin(x).backward(dy)
    pruned = layers._pruned(dy, 0.7, 0)
    assert abs(float((pruned == 0).float().mean()) - 0.7) < 0.02
    plain(x).backward(pruned)
    assert torch.equal(lin.weight.grad, plain.weight.grad)


def test_embedding_module(layers):
    emb = layers.Embedding(50, 40, scale=2.0, padding_idx=3, out_dtype=torch.float32, device="cuda")
    ids = torch.tensor([[1, 3, 49], [1, 1, 0]], device="cuda")
    out = emb(ids)
    assert out.shape == (2, 3, 40) and torch.equal(out, 2.0 * emb.weight[ids])
    out.sum().backward()
    want = torch.zeros(50, device="cuda")
    want[1], want[49], want[0] = 6.0, 2.0, 2.0
    assert torch.equal(emb.weight.grad, want[:, None].expand(50, 40))


def test_clipper_needs_gradients(layers):
    with pytest.raises(ValueError):
        layers.GradClipper([torch.nn.Parameter(torch.zeros(3, device="cuda"))], 1.0)


def test_clipper_notices_replaced_gradients(layers):
    p = torch.nn.Parameter(torch.zeros(3, device="cuda"))
    p.grad = torch.full((3,), 2.0, device="cuda")
    c = layers.GradClipper([p], 1.0)
    norm = float(c.clip())
    assert abs(norm - 12 ** 0.5) < 1e-5 and abs(float(p.grad.norm()) - 1.0) < 1e-5
    p.grad = torch.ones(3, device="cuda")
    with pytest.raises(RuntimeError):
        c.clip()


def test_only_the_gradients_asked_for(layers):
    lin = layers.Fp8Linear(64, 32, device="cuda")
    x = torch.randn(7, 64, device="cuda").bfloat16()
    lin(x).sum().backward()                                       # the input needs none
    assert lin.weight.grad is not None
    want = lin.weight.grad.clone()
    lin.weight.grad = None
    x.requires_grad_()
    lin(x).sum().backward()
    assert torch.equal(want, lin.weight.grad) and x.grad is not None
    lin.weight.requires_grad_(False)
    once = x.grad.clone()
    x.grad = None
    lin(x).sum().backward()
    assert torch.equal(once, x.grad)


def test_example_learns(lgn):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import lm_step
        losses, norms = lm_step.train(steps=40, tokens=1024)
    finally:
        sys.path.pop(0)
    assert all(np.isfinite(losses)) and all(np.isfinite(norms)) and min(norms) > 0
    assert np.mean(losses[-5:]) < 0.75 * np.mean(losses[:5])
