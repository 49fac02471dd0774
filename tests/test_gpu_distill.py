"""The loss against a teacher's top logits and its gradient, against fp64.

Bounds, in units of 2^-24: an exponential of a value x below the maximum is off by 4 (base-2 approximation, 2^-22) + 3 |x|
(argument: difference, scale, product); a sum by its terms' mean error and the longest chain of additions (64 values in a
thread, 5 shuffles, 8 warps, 8 CTAs; chunks of longer rows add 64 each).  A softmax value is therefore off by less than 400 + 3 |x|
relative, which bounds the gradient before its rounding; the loss adds logarithms of such sums and a mean of differences
of logits, both weighted as in its formula."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def reference(s, ids, z, labels, temp, alpha, weight):
    """(loss, its bound, gradient, its bound) in fp64."""
    s, z, ids = s.double(), z.double(), ids.long()
    t, v = s.shape
    there = (ids >= 0) & (ids < v) & (z != -float("inf")) & (alpha > 0)
    some = there.any(1)
    at = torch.where(there, ids, 0)
    zt = torch.where(there, z / temp, -float("inf"))
    p = torch.where(some[:, None], torch.softmax(zt, 1), 0.0).nan_to_num(0.0) if ids.shape[1] else torch.zeros(t, 0, dtype=torch.float64, device=s.device)
    logp = torch.where(p > 0, torch.log(p), 0.0)
    logq, logq1 = torch.log_softmax(s / temp, 1), torch.log_softmax(s, 1)
    picked = logq.gather(1, at)
    loss = alpha * temp ** 2 * torch.where(p > 0, p * (logp - picked), 0.0).sum(1)
    dense = torch.zeros_like(s).scatter_add_(1, at, p)
    known = torch.zeros(t, dtype=torch.bool, device=s.device)
    onehot = torch.zeros_like(s)
    spread = torch.where(p > 0, p * (logp.abs() + picked.abs()), 0.0).sum(1)
    bound = alpha * temp ** 2 * some * (800 + 20 * spread) * U
    if labels is not None and alpha < 1:
        lab = labels.long()
        known = (lab >= 0) & (lab < v)
        lab = torch.where(known, lab, 0)
        onehot.scatter_(1, lab[:, None], known.double()[:, None])
        ce = torch.where(known, -logq1.gather(1, lab[:, None])[:, 0], 0.0)
        loss, bound = loss + (1 - alpha) * ce, bound + (1 - alpha) * known * (400 + 20 * ce.abs()) * U
    bound = bound + 4 * U * loss.abs()
    w = torch.ones(t, dtype=torch.float64, device=s.device) if weight is None else weight.double()
    kt, k1 = (w * alpha * temp * some)[:, None], (w * (1 - alpha) * known)[:, None]
    live = (some | known)[:, None]
    q, q1 = (torch.where(live, torch.exp(a), 0.0) for a in (logq, logq1))
    d = kt * (q - dense) + k1 * (q1 - onehot)
    far, far1 = (torch.where(q > 0, -logq, 0.0).clamp(max=90.0), torch.where(q1 > 0, -logq1, 0.0).clamp(max=90.0))
    zfar = float((zt.amax(1, keepdim=True) - zt)[there].max()) if there.any() else 0.0
    dbound = (kt * (q * (400 + 3 * far) + dense * (400 + 3 * min(zfar, 90.0))) + k1 * (q1 * (400 + 3 * far1) + 4 * onehot)) * U + 2.0 ** -120
    return loss, bound, d, dbound


def check(got, want, bound):
    tol = bound + HALF[got.dtype] * (want.abs() + bound)
    same = (got.isnan() & want.isnan()) | (got.double() == want)
    bad = ~((got.double() - want).abs() <= tol) & ~same
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4], got[bad][:4], want[bad][:4])


def inputs(t, v, top, seed, dtype=torch.float32, zt=torch.float32, it=torch.int64):
    g = torch.Generator().manual_seed(seed)
    s = 3.0 * torch.randn(t, v, generator=g)
    ids = torch.randint(-1, v, (t, top), generator=g)
    ids[torch.rand(t, generator=g) < 0.1] = -1
    z = 4.0 * torch.randn(t, top, generator=g)
    labels = torch.randint(0, v, (t,), generator=g)
    if top:
        labels = torch.where(torch.rand(t, generator=g) < 0.5, ids[:, 0], labels)
    labels[torch.rand(t, generator=g) < 0.2] = -100
    weight = torch.rand(t, generator=g)
    return s.to(dtype).cuda(), ids.to(it).cuda(), z.to(zt).cuda(), labels.to(it).cuda(), weight.cuda()


def check_call(lgn, s, ids, z, labels, temp, alpha, weight):
    loss, bound, d, dbound = reference(s, ids, z, labels, temp, alpha, weight)
    got, none = lgn.lgn_distill_loss(s, ids, z, labels, temp, alpha, weight)
    assert none is None
    check(got, loss, bound)
    got, grad = lgn.lgn_distill_loss(s, ids, z, labels, temp, alpha, weight, grad=True)
    check(got, loss, bound)
    check(grad, d, dbound)
    return grad


SHAPES = [(1, 1, 1), (3, 7, 2), (5, 1000, 17), (2, 8191, 64), (2, 8192, 64), (4, 8200, 33), (300, 640, 5), (7, 50021, 100), (3, 131072, 256), (160, 33000, 8), (2, 300000, 8), (40, 4099, 1024), (3, 500, 0)]


@pytest.mark.parametrize("temp,alpha,labelled", [(1.0, 1.0, False), (1.0, 0.4, True), (2.5, 0.3, True), (0.7, 1.0, True), (3.0, 0.0, True), (1.5, 0.6, False)])
@pytest.mark.parametrize("dtype,zt,it", [("f32", "f32", torch.int64), ("bf16", "bf16", torch.int32)])
@pytest.mark.parametrize("t,v,top", SHAPES)
def test_loss_and_gradient(lgn, t, v, top, dtype, zt, it, temp, alpha, labelled):
    s, ids, z, labels, weight = inputs(t, v, top, t + v + top, DT[dtype], DT[zt], it)
    check_call(lgn, s, ids, z, labels if labelled else None, temp, alpha, weight if t % 2 else None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks(lgn, dtype):
    """Rows without a teacher, without a label, without either; masked logits of -inf and of the type's lowest value; masked teacher's logits;
    places outside the vocabulary; the same place named several times and as the label."""
    s, ids, z, labels, weight = inputs(12, 3000, 20, 5, DT[dtype])
    ids[0], labels[0] = -1, 4
    ids[1], labels[1] = 3000, -1
    ids[2], labels[2] = torch.arange(20), 3000
    z[3] = -float("inf")
    z[4, 1:] = -float("inf")
    ids[5, :10], labels[5] = 77, 77
    ids[6] = 2999
    s[7, 100:] = -float("inf"); ids[7] = torch.arange(20) * 3; labels[7] = 50
    s[8, 5:] = torch.finfo(DT[dtype]).min; ids[8] = torch.arange(20) % 5; labels[8] = 0
    z[9, 1:] = torch.finfo(torch.float32).min
    ids[10] = 2 ** 40
    for temp, alpha in ((1.0, 0.5), (2.0, 0.5), (0.5, 1.0), (1.0, 0.0)):
        check_call(lgn, s, ids, z, labels, temp, alpha, weight)


@pytest.mark.parametrize("v", [900, 40000])
def test_values_that_are_not_finite(lgn, v):
    s, ids, z, labels, weight = inputs(8, v, 6, 6)
    ids[:] = torch.arange(6) * 3
    s[0, 5] = float("nan"); s[1, 7] = float("inf"); s[2] = -float("inf")
    s[3, 6] = -float("inf")                               # a place with p > 0 that the student rules out
    s[4] = float("nan"); ids[4], labels[4] = -1, -1
    z[5, 2] = float("nan")
    labels[0:3] = 1
    loss, grad = lgn.lgn_distill_loss(s, ids, z, labels, 1.0, 0.5, weight, grad=True)
    assert loss[:3].isnan().all() and grad[:3].isnan().all()
    assert loss[3] == float("inf") and grad[3].isfinite().all()
    assert loss[4] == 0 and (grad[4] == 0).all()
    assert loss[5].isnan()
    keep = torch.tensor([3, 6, 7], device="cuda")
    _, _, d, dbound = reference(s[keep], ids[keep], z[keep], labels[keep], 1.0, 0.5, weight[keep])
    check(grad[keep], d, dbound)
    assert loss[6:].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [1001, 20000, 140001])
def test_views_in_place_and_given_outputs(lgn, v, dtype):
    """Rows at odd addresses, gradients over the logits or aligned differently; what lies around stays."""
    s, ids, z, labels, weight = inputs(5, v + 9, 12, 7, DT[dtype])
    ids = torch.where(ids >= v, -1, ids)
    labels = torch.where(labels >= v, -1, labels)
    wide_ids, wide_z = torch.full((5, 20), 1, device="cuda"), torch.zeros(5, 31, device="cuda")
    wide_ids[:, 3:15], wide_z[:, 7:19] = ids, z
    for lo in (0, 1, 8, 3):
        view = s[:, lo:lo + v]
        loss, bound, d, dbound = reference(view, ids, z, labels, 1.3, 0.5, weight)
        for shift in (0, 1, 4):
            whole = torch.full((7, v + 11), -5.0, dtype=DT[dtype], device="cuda")
            out, per_row = whole[1:6, shift:shift + v], torch.full((7,), -5.0, device="cuda")
            got, same = lgn.lgn_distill_loss(view, wide_ids[:, 3:15], wide_z[:, 7:19], labels, 1.3, 0.5, weight, loss=per_row[1:6], dlogits=out)
            assert same is out
            check(got, loss, bound)
            check(out, d, dbound)
            out.fill_(-5.0); got.fill_(-5.0)
            assert (whole == -5.0).all() and (per_row == -5.0).all()
        copy = s.clone()
        place = copy[:, lo:lo + v]
        _, same = lgn.lgn_distill_loss(place, ids, z, labels, 1.3, 0.5, weight, dlogits=place)
        check(place, d, dbound)
        place.copy_(view)
        assert torch.equal(copy, s)


def test_gradient_against_differences(lgn):
    """(loss(s + h e) - loss(s - h e)) / 2h of the fp64 form and of the kernel's loss; the kernel's own is off by its loss's bound over h."""
    s, ids, z, labels, _ = inputs(6, 50, 4, 11)
    h = 2.0 ** -6
    _, grad = lgn.lgn_distill_loss(s, ids, z, labels, 1.7, 0.6, grad=True)
    for i in range(0, 50, 7):
        up, down = s.clone(), s.clone()
        up[:, i] += h
        down[:, i] -= h
        a, _ = lgn.lgn_distill_loss(up, ids, z, labels, 1.7, 0.6)
        b, _ = lgn.lgn_distill_loss(down, ids, z, labels, 1.7, 0.6)
        _, bound, _, _ = reference(s, ids, z, labels, 1.7, 0.6, None)
        # third derivatives of a log-sum-exp are below 1/2 per temperature: h^2 / 6 of that times the weights alpha T + 1
        tol = 2 * bound / (2 * h) + h * h / 6 * (0.6 * 1.7 + 1.0) + 2 * bound
        assert (((a - b).double() / (2 * h) - grad[:, i].double()).abs() <= tol).all()


def test_empty(lgn):
    s, ids, z, labels, weight = inputs(3, 5, 2, 1)
    loss, grad = lgn.lgn_distill_loss(s[:0], ids[:0], z[:0], labels[:0], weight=weight[:0], grad=True)
    assert loss.shape == (0,) and grad.shape == (0, 5)
    loss, grad = lgn.lgn_distill_loss(s[:, :0], ids, z, grad=True)
    assert (loss == 0).all() and grad.shape == (3, 0)


def test_streams_graphs_and_the_same_bits(lgn):
    s, ids, z, labels, weight = inputs(64, 30000, 40, 2, torch.bfloat16)
    first = lgn.lgn_distill_loss(s, ids, z, labels, 2.0, 0.5, weight, grad=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = lgn.lgn_distill_loss(s, ids, z, labels, 2.0, 0.5, weight, grad=True, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = lgn.lgn_distill_loss(s, ids, z, labels, 2.0, 0.5, weight, grad=True)
    for _ in range(3):
        graph.replay()
        for got in (other, captured):
            assert torch.equal(got[0], first[0]) and torch.equal(got[1], first[1])


def test_two_threads(lgn):
    """Calls whose CTAs need different amounts of shared memory, from two threads at once."""
    import threading
    sets = [inputs(8, 16000, top, top, torch.bfloat16) for top in (1024, 700)]
    want = [lgn.lgn_distill_loss(s, ids, z, labels, 2.0, 0.5, grad=True) for s, ids, z, labels, _ in sets]
    wrong = []

    def run(i):
        s, ids, z, labels, _ = sets[i]
        stream = torch.cuda.Stream()
        try:
            for _ in range(3000):
                loss, d = lgn.lgn_distill_loss(s, ids, z, labels, 2.0, 0.5, grad=True, stream=stream)
            stream.synchronize()
            if not (torch.equal(loss, want[i][0]) and torch.equal(d, want[i][1])):
                wrong.append(i)
        except Exception as e:
            wrong.append(e)
    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong
