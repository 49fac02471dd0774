"""Global norm and clipping against fp64.

The sum adds squares in fp32 over at most 16 values (each addition and each product off by at most 2^-24 of
the terms so far, all of one sign: 17 * 2^-24 relative) and in fp64 beyond; the norm halves that and is
rounded to fp32.  A clipped value: coefficient (norm's error, one fp32 rounding), one product, one rounding."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
NORM_TOL = 0.5 * 17 * 2.0 ** -24 + 2.0 ** -24


def np64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def make(sizes, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(scale * torch.randn(n, generator=g)).to(torch.bfloat16 if i % 3 == 1 else torch.float32).cuda() for i, n in enumerate(sizes)]


def true_norm(ts):
    return math.sqrt(sum(float((np64(t) ** 2).sum()) for t in ts))


def check(lgn, ts, outs, before, max_norm, rec):
    norm = true_norm(before)
    r = lgn.read_norm_record(rec)
    assert abs(r["norm"] - norm) <= NORM_TOL * norm
    assert abs(math.sqrt(r["sum_sq"]) - norm) <= NORM_TOL * norm
    coef = max_norm / norm if norm > max_norm else 1.0
    assert abs(r["coef"] - coef) <= (NORM_TOL + 2.0 ** -24) * coef
    assert r["n_nonfinite"] == 0
    for b, o in zip(before, outs):
        want = np64(b) * coef
        tol = (NORM_TOL + 2 * 2.0 ** -24 + HALF[o.dtype]) * (1 + 2.0 ** -7) * np.abs(want) + 2.0 ** -149
        assert np.all(np.abs(np64(o) - want) <= tol)


LISTS = [[1], [0, 3, 0], [7, 8, 9, 15, 16, 17, 31, 32, 33], [8191, 8192, 8193, 16383, 16385], [100003, 1, 50001, 2, 2000000],
         [5] * 200, [17 + i % 50 for i in range(700)], [1000] * 1100]


@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("ratio", [0.5, 3.0])
def test_clip_in_and_out_of_place(lgn, sizes, ratio):
    before = make(sizes, len(sizes))
    max_norm = true_norm(before) / ratio
    rec, ws = lgn.new_norm_record("cuda"), lgn.new_clip_workspace("cuda", len(sizes))
    ws.fill_(0xEE)
    outs = [torch.full_like(t, 9.0) for t in before]
    lgn.lgn_clip_grad_norm(lgn.make_grads(before, outs), max_norm, rec, ws)
    check(lgn, before, outs, before, max_norm, rec)
    place = [t.clone() for t in before]
    lgn.lgn_clip_grad_norm(lgn.make_grads(place), max_norm, rec, ws)
    for a, b in zip(place, outs):
        assert torch.equal(a, b)
    if ratio < 1:
        for a, b in zip(place, before):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_pieces_of_one_buffer(lgn, dtype):
    """Tensors at every element offset of a larger buffer, inputs and outputs aligned alike or not; what lies
    between them is not touched."""
    buf = torch.randn(200000, device="cuda").to(dtype)
    for shift in (0, 1, 5):
        out = torch.full((200100,), 9.0, device="cuda", dtype=dtype)
        at, ts, os_, spans = 0, [], [], []
        for i in range(40):
            n = 1 + (i * 379) % 9000
            ts.append(buf[at:at + n])
            os_.append(out[at + shift:at + shift + n])
            spans.append((at + shift, at + shift + n))
            at += n + 1 + i % 3
        rec, ws = lgn.new_norm_record("cuda"), lgn.new_clip_workspace("cuda")
        lgn.lgn_clip_grad_norm(lgn.make_grads(ts, os_), 2.0, rec, ws)
        check(lgn, ts, os_, ts, 2.0, rec)
        mask = torch.ones(200100, dtype=torch.bool, device="cuda")
        for a, b in spans:
            mask[a:b] = False
        assert bool((out[mask] == 9.0).all())


@pytest.mark.parametrize("value", [1e-30, 1e-38, 1e-42, 1e25, 3e38])
def test_range(lgn, value):
    """Squares that leave fp32's range on either side."""
    t = torch.full((5001,), value, device="cuda")
    rec, ws = lgn.new_norm_record("cuda"), lgn.new_clip_workspace("cuda")
    lgn.lgn_grad_norm(lgn.make_grads([t]), rec, ws)
    r = lgn.read_norm_record(rec)
    want = float(t[0].double()) * math.sqrt(5001)
    assert abs(math.sqrt(r["sum_sq"]) - want) <= NORM_TOL * want
    assert r["coef"] == 1.0
    if want < 3.4e38:
        assert abs(r["norm"] - want) <= NORM_TOL * want + 2.0 ** -149
    else:
        assert math.isinf(r["norm"])


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), float("-inf")])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_non_finite_values_are_counted_and_nothing_is_scaled(lgn, bad, dtype):
    a, b = torch.randn(70001, device="cuda").to(dtype), torch.randn(33, device="cuda").to(dtype)
    a[0] = a[70000] = b[17] = bad
    before = [a.clone(), b.clone()]
    rec, ws = lgn.new_norm_record("cuda"), lgn.new_clip_workspace("cuda")
    lgn.lgn_clip_grad_norm(lgn.make_grads([a, b]), 0.1, rec, ws)
    r = lgn.read_norm_record(rec)
    assert r["n_nonfinite"] == 3 and not math.isfinite(r["norm"]) and r["coef"] == 1.0
    for x, y in zip((a, b), before):
        assert torch.equal(x.isnan(), y.isnan()) and torch.equal(x.nan_to_num(), y.nan_to_num())


def test_zero_and_limits(lgn):
    rec, ws = lgn.new_norm_record("cuda"), lgn.new_clip_workspace("cuda")
    z = torch.zeros(1000, device="cuda")
    lgn.lgn_clip_grad_norm(lgn.make_grads([z]), 1.0, rec, ws)
    assert lgn.read_norm_record(rec) == {"norm": 0.0, "coef": 1.0, "n_nonfinite": 0, "sum_sq": 0.0}
    lgn.lgn_clip_grad_norm(lgn.make_grads([]), 1.0, rec, ws)
    assert lgn.read_norm_record(rec)["sum_sq"] == 0.0
    t = torch.randn(1000, device="cuda")
    keep = t.clone()
    lgn.lgn_clip_grad_norm(lgn.make_grads([t]), math.inf, rec, ws)
    assert torch.equal(t, keep)
    lgn.lgn_clip_grad_norm(lgn.make_grads([t]), 0.0, rec, ws)
    assert bool((t == 0).all())


def test_shards_add_their_sums(lgn):
    """lgn_grad_norm on two shards, their sums added (what ranks all-reduce), lgn_clip_apply on each: the same
    as one call over both."""
    ts = make([50001, 777, 12345, 64], 5)
    ws = lgn.new_clip_workspace("cuda")
    recs = [lgn.new_norm_record("cuda") for _ in range(3)]
    shards = [[t.clone() for t in ts[:2]], [t.clone() for t in ts[2:]]]
    for s, r in zip(shards, recs):
        lgn.lgn_grad_norm(lgn.make_grads(s), r, ws)
    both = lgn.sum_sq_of(recs[0]) + lgn.sum_sq_of(recs[1])
    for s, r in zip(shards, recs):
        lgn.sum_sq_of(r).copy_(both)
        lgn.lgn_clip_apply(lgn.make_grads(s), 1.5, r)
    whole = [t.clone() for t in ts]
    lgn.lgn_clip_grad_norm(lgn.make_grads(whole), 1.5, recs[2], ws)
    a, b = lgn.read_norm_record(recs[0]), lgn.read_norm_record(recs[2])
    assert abs(a["norm"] - b["norm"]) <= 2 * NORM_TOL * b["norm"]
    for x, y in zip(shards[0] + shards[1], whole):
        assert np.all(np.abs(np64(x) - np64(y)) <= 2 * (NORM_TOL + 2.0 ** -24 + HALF[x.dtype]) * np.abs(np64(y)))


def test_same_bits_and_other_streams(lgn):
    ts = make([100003, 1, 50001], 8)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    seen = []
    for _ in range(4):
        rec, ws = lgn.new_norm_record("cuda"), lgn.new_clip_workspace("cuda")
        s.wait_stream(torch.cuda.current_stream())
        outs = [torch.empty_like(t) for t in ts]
        lgn.lgn_clip_grad_norm(lgn.make_grads(ts, outs), 1.0, rec, ws, stream=s)
        s.synchronize()
        seen.append((lgn.read_norm_record(rec), outs))
    for r, o in seen[1:]:
        assert r == seen[0][0] and all(torch.equal(x, y) for x, y in zip(o, seen[0][1]))


def test_tensor_beyond_32_bits(lgn):
    n = 2 ** 32 + 37
    t = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    t[0], t[2 ** 31], t[n - 1] = 3.0, 4.0, 12.0
    rec, ws = lgn.new_norm_record("cuda"), lgn.new_clip_workspace("cuda")
    lgn.lgn_clip_grad_norm(lgn.make_grads([t]), 6.5, rec, ws)
    r = lgn.read_norm_record(rec)
    assert r["sum_sq"] == 169.0 and r["norm"] == 13.0 and r["coef"] == 0.5
    assert [float(t[i]) for i in (0, 2 ** 31, n - 1)] == [1.5, 2.0, 6.0]


def test_refusals(lgn):
    t = torch.zeros(100, device="cuda")
    rec, ws = lgn.new_norm_record("cuda"), lgn.new_clip_workspace("cuda", 3)
    g = lgn.make_grads([t])
    with pytest.raises(lgn.LgnError):
        lgn.lgn_clip_grad_norm(g, float("nan"), rec, ws)
    with pytest.raises(lgn.LgnError):
        lgn.lgn_clip_grad_norm(g, -1.0, rec, ws)
    with pytest.raises(lgn.LgnError) as e:
        lgn.lgn_clip_grad_norm(g, 1.0, rec, ws[:64])
    assert e.value.code == 3
    with pytest.raises(lgn.LgnError):
        lgn.lgn_clip_grad_norm(lgn.make_grads([t[:50]], [t[20:70]]), 1.0, rec, ws)
    with pytest.raises(TypeError):
        lgn.make_grads([t.half()])
    with pytest.raises(ValueError):
        lgn.make_grads([t], [t[:50]])
    with pytest.raises(ValueError):
        lgn.make_grads([t[::2]])
    with pytest.raises(ValueError):
        lgn.lgn_grad_norm(g, rec[:8], ws)
    assert lgn.raw().lgn_clip_workspace_bytes(-1) == 0
    assert lgn.raw().lgn_grad_norm(None, 1, rec.data_ptr(), ws.data_ptr(), ws.numel(), None) == 1
