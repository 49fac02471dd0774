"""Int8Linear, ExpertLinear, by_expert and DistillLoss as torch modules, and the example that runs them together."""
import os
import sys

import pytest
import torch

from fp8_helpers import quantise, to_np
from test_gpu_distill import check as check_bound, inputs, reference as distill_reference
from test_gpu_grouped import check as check_grouped, forward as grouped_forward, gradient as grouped_gradient
from test_gpu_int8 import reference as int8_reference

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def layers(lgn):
    from paper_2006_08173_b200 import layers as mod
    return mod


def check_int8(y, x, w):
    (a, sa), (b, sb) = int8_reference(x.detach()), int8_reference(w.detach())
    want = ((a @ b.t()) * sa.double()[:, None] * sb.double()).cuda()                    # whole numbers: the sums are exact
    half = 2.0 ** -8 if y.dtype == torch.bfloat16 else 0.0
    assert bool(((y.double() - want).abs() <= want.abs() * (3.001 * 2.0 ** -24 + 1.001 * half)).all())


def fp8(t, fmt, square=False):
    return torch.from_numpy(quantise(to_np(t), fmt, square)[0]).cuda()


def check_fp8(got, a, b, k):
    """Groups of 32 added in fp32, one rounding."""
    want, mag = a @ b, a.abs() @ b.abs()
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    tol = ((k + 31) // 32 + 32) * 2.0 ** -23 * mag
    assert bool(((got.double() - want).abs() <= tol + half * (want.abs() + tol)).all())


@pytest.mark.parametrize("t,k,n,dtype", [(1, 64, 40, torch.bfloat16), (37, 300, 129, torch.float32), (200, 256, 512, torch.bfloat16)])
def test_int8_linear(layers, t, k, n, dtype):
    torch.manual_seed(t)
    lin = layers.Int8Linear(k, n, device="cuda")
    x = torch.randn(t, k, device="cuda").to(dtype).requires_grad_()
    dy = (1e-4 * torch.randn(t, n, device="cuda")).to(dtype)
    y = lin(x)
    y.backward(dy)
    check_int8(y.detach(), x, lin.weight)
    check_fp8(x.grad, fp8(dy, 1), fp8(lin.weight, 0, True), n)
    check_fp8(lin.weight.grad, fp8(dy.t().contiguous(), 1), fp8(x.t().contiguous(), 0).t(), t)
    lin.check()
    lin.freeze()
    with torch.no_grad():
        assert torch.equal(lin(x), y)
        lin.weight.zero_()
        assert torch.equal(lin(x), y)                              # as of freeze()
    with pytest.raises(RuntimeError):
        lin(x)
    lin.freeze(False)
    assert not lin(x).any()


@pytest.mark.parametrize("needs", [(True, False), (False, True), (False, False)])
def test_gradients_that_are_not_asked_for(layers, needs):
    lin, mix = layers.Int8Linear(64, 48, device="cuda"), layers.ExpertLinear(3, 64, 48, device="cuda")
    offsets = torch.tensor([0, 5, 5, 9], device="cuda")
    for layer, args in ((lin, ()), (mix, (offsets,))):
        x = torch.randn(9, 64, device="cuda", requires_grad=needs[0])
        layer.weight.requires_grad_(needs[1])
        y = layer(x, *args)
        if any(needs):
            y.sum().backward()
        assert (x.grad is not None, layer.weight.grad is not None) == needs


def test_pruned_gradients(layers, lgn):
    """The gradients of a pruned layer are those of the pruned gradient."""
    torch.manual_seed(0)
    offsets = torch.tensor([0, 200, 512], device="cuda")
    for make, args in ((lambda s: layers.Int8Linear(128, 256, sparsity=s, device="cuda", seed=9), ()), (lambda s: layers.ExpertLinear(2, 128, 256, sparsity=s, device="cuda", seed=9), (offsets,))):
        lin, plain = make(0.7), make(0.0)
        plain.weight.data.copy_(lin.weight.data)
        x = torch.randn(512, 128, device="cuda").bfloat16()
        dy = torch.exp(-12 + 2 * torch.randn(512, 256, device="cuda")).bfloat16()
        a, b = x.clone().requires_grad_(), x.clone().requires_grad_()
        lin(a, *args).backward(dy)
        plain(b, *args).backward(layers._pruned(dy, 0.7, 9))
        assert torch.equal(a.grad, b.grad) and torch.equal(lin.weight.grad, plain.weight.grad)
        lin.check()


@pytest.mark.parametrize("experts,rows,k,n,dtype", [(1, 7, 24, 40, torch.float32), (5, 300, 72, 136, torch.bfloat16), (64, 500, 33, 50, torch.float32)])
def test_experts(layers, experts, rows, k, n, dtype):
    torch.manual_seed(rows)
    mix = layers.ExpertLinear(experts, k, n, device="cuda")
    ids = torch.randint(-1, experts + 1, (rows,), device="cuda")                        # some belong to no expert
    order, offsets = layers.by_expert(ids, experts)
    ends = offsets.tolist()
    assert all((ids[order[ends[e]:ends[e + 1]]] == e).all() for e in range(experts)) and ends[0] == int((ids < 0).sum())
    assert all((order[ends[e]:ends[e + 1]].diff() > 0).all() for e in range(experts))
    x = torch.randn(rows, k, device="cuda").to(dtype)[order].requires_grad_()
    dy = (1e-3 * torch.randn(rows, n, device="cuda")).to(dtype)
    y = mix(x, offsets)
    y.backward(dy)
    xb, wb, db = x.detach().bfloat16(), mix.weight.detach().bfloat16(), dy.bfloat16()
    check_grouped(y.detach(), *grouped_forward(xb, wb, ends, False), k)
    check_grouped(x.grad, *grouped_forward(db, wb, ends, True), n)
    check_grouped(mix.weight.grad, *grouped_gradient(db, xb, ends), rows)
    outside = torch.cat([torch.arange(0, ends[0]), torch.arange(ends[-1], rows)]).cuda()
    assert not y[outside].any() and not x.grad[outside].any()
    mix.check()


@pytest.mark.parametrize("dtype,shape", [(torch.float32, (6,)), (torch.bfloat16, (2, 3))])
@pytest.mark.parametrize("labelled", [False, True])
def test_distill_loss(layers, dtype, shape, labelled):
    s, ids, z, labels, _ = inputs(6, 500, 8, 3, dtype)
    labels = labels if labelled else None
    up = torch.rand(6, device="cuda")
    leaf = s.reshape(*shape, 500).clone().requires_grad_()
    loss = layers.DistillLoss(2.0, 0.6)(leaf, ids.reshape(*shape, 8), z.reshape(*shape, 8), None if labels is None else labels.reshape(shape))
    assert loss.shape == shape
    loss.backward(up.reshape(shape))
    want, bound, d, dbound = distill_reference(s, ids, z, labels, 2.0, 0.6, up)
    check_bound(loss.detach().reshape(6), want, bound)
    check_bound(leaf.grad.reshape(6, 500), d, dbound)
    strided = torch.zeros(500, 6, device="cuda", dtype=dtype).copy_(s.t()).t().requires_grad_()      # transposed logits, an expanded upstream gradient
    layers.DistillLoss(2.0, 0.6)(strided, ids, z, labels).sum().backward()
    _, _, d, dbound = distill_reference(s, ids, z, labels, 2.0, 0.6, None)
    check_bound(strided.grad, d, dbound)


@pytest.mark.parametrize("sparsity", [0.0, 0.5])
def test_example_runs(sparsity):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import distill_step
    losses, norms = distill_step.train(steps=3, sparsity=sparsity)
    assert len(losses) == 3 and all(0.0 < v < 1e6 for v in losses) and all(0.0 < v < 1e6 for v in norms)


def test_gradients_along_the_example(layers):
    """One step of the example's student; every gradient is the formula's of what the module next to it saw."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import distill_step
    torch.manual_seed(1)
    model = distill_step.Student(300, 64, 80, 6, 2, 0.0)
    seen = {}

    def keep(name):
        def hook(module, args, out):
            seen[name] = (args, out)
            out.retain_grad()
            if args[0].requires_grad:
                args[0].retain_grad()
        return hook
    for name in ("up", "down", "head"):
        getattr(model, name).register_forward_hook(keep(name))
    places = torch.stack([torch.randperm(300)[:8] for _ in range(90)]).cuda()
    z, labels = torch.randn(90, 8, device="cuda"), torch.randint(0, 300, (90,), device="cuda")
    layers.DistillLoss(2.0, 0.5)(model(torch.randint(0, 300, (90,), device="cuda")), places, z, labels).sum().backward()
    (x,), logits = seen["head"]
    check_int8(logits.detach(), x, model.head.weight)
    _, _, d, dbound = distill_reference(logits.detach(), places, z, labels, 2.0, 0.5, None)
    check_bound(logits.grad, d, dbound)
    check_fp8(model.head.weight.grad, fp8(logits.grad.t().contiguous(), 1), fp8(x.detach().t().contiguous(), 0).t(), 90)
    check_fp8(x.grad, fp8(logits.grad, 1), fp8(model.head.weight, 0, True), 300)
    for name in ("up", "down"):
        (x, offsets), y = seen[name]
        layer, ends = getattr(model, name), offsets.tolist()
        check_grouped(y.detach(), *grouped_forward(x.detach().bfloat16(), layer.weight.detach().bfloat16(), ends, False), x.shape[1])
        check_grouped(layer.weight.grad, *grouped_gradient(y.grad.bfloat16(), x.detach().bfloat16(), ends), x.shape[0])
        check_grouped(x.grad, *grouped_forward(y.grad.bfloat16(), layer.weight.detach().bfloat16(), ends, True), y.shape[1])
    assert bool(model.embed.weight.grad.any()) and bool(model.gate.weight.grad.any())


def test_frozen_layers_refuse_every_gradient(layers):
    """A layer that comes first in a model: its input wants no gradient, its weights do."""
    lin = layers.Int8Linear(64, 48, device="cuda")
    x = torch.randn(9, 64, device="cuda")
    lin.freeze()
    with pytest.raises(RuntimeError):
        lin(x)
    lin.weight.requires_grad_(False)
    y = lin(x)
    with pytest.raises(RuntimeError):
        lin(x.clone().requires_grad_())
    with torch.inference_mode():
        assert torch.equal(lin(x), y)


def test_first_pass_in_inference_mode(layers):
    """check() after it, and passes that train."""
    lin, mix, fp8_lin = layers.Int8Linear(64, 48, device="cuda"), layers.ExpertLinear(2, 64, 48, device="cuda"), layers.Fp8Linear(64, 48, device="cuda")
    offsets = torch.tensor([0, 4, 9], device="cuda")
    x = torch.randn(9, 64, device="cuda")
    for layer, args in ((lin, ()), (mix, (offsets,)), (fp8_lin, ())):
        with torch.inference_mode():
            y = layer(x, *args)
        layer.check()
        z = layer(x, *args)
        z.sum().backward()
        layer.check()
        assert torch.equal(y, z) and layer.weight.grad is not None


def test_rows_of_no_expert_do_not_reach_the_pruning(layers):
    torch.manual_seed(0)
    lin, plain = (layers.ExpertLinear(2, 128, 256, sparsity=s, device="cuda", seed=9) for s in (0.7, 0.0))
    plain.weight.data.copy_(lin.weight.data)
    offsets = torch.tensor([40, 200, 400], device="cuda")
    x = torch.randn(512, 128, device="cuda").bfloat16()
    dy = torch.exp(-12 + 2 * torch.randn(512, 256, device="cuda")).bfloat16()
    dy[:40], dy[400:] = float("nan"), float("inf")
    zeros = dy.clone()
    zeros[:40], zeros[400:] = 0.0, 0.0
    a, b = x.clone().requires_grad_(), x.clone().requires_grad_()
    lin(a, offsets).backward(dy)
    plain(b, offsets).backward(layers._pruned(zeros, 0.7, 9))
    assert torch.equal(a.grad, b.grad) and torch.equal(lin.weight.grad, plain.weight.grad)
    assert bool(a.grad.isfinite().all()) and bool(lin.weight.grad.isfinite().all())
    lin.check()


@pytest.mark.parametrize("sparsity", [0.0, 0.5])
def test_captured_step(layers, sparsity):
    """A training step captured once and replayed on other tokens, whose experts have other numbers of rows, gives what the same step gives directly."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import distill_step
    torch.manual_seed(2)
    model = distill_step.Student(300, 64, 80, 6, 2, sparsity)
    loss_of = layers.DistillLoss(2.0, 0.5)
    tokens = torch.randint(0, 300, (90,), device="cuda")
    places = torch.stack([torch.randperm(300)[:8] for _ in range(90)]).cuda()
    z, labels = torch.randn(90, 8, device="cuda"), torch.randint(0, 300, (90,), device="cuda")

    def step():
        for q in model.parameters():
            q.grad = None
        loss = loss_of(model(tokens), places, z, labels)
        loss.sum().backward()
        return loss.detach()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = step()
    held = [(n, q.grad) for n, q in model.named_parameters()]
    for seed in range(3):
        torch.manual_seed(seed)
        tokens.copy_(torch.randint(0, 300 if seed else 2, (90,)))
        z.normal_()
        graph.replay()
        got = [loss.clone()] + [g.clone() for _, g in held]
        want = [step()] + [q.grad for q in model.parameters()]
        for name, a, b in zip(["loss"] + [n for n, _ in held], got, want):
            if name in ("gate.weight", "embed.weight"):                # products of torch lead to them
                assert bool(((a - b).abs() <= 1e-4 * b.abs().max()).all())
            else:
                assert torch.equal(a, b), name
    for m in (model.up, model.down, model.head):
        m.check()
