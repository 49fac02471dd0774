"""Norm and clipping of more than 18 MiB of gradients, where a CTA takes several tiles and the last one adds the partial sums: every value
of dense random tensors, in place, to outputs aligned otherwise, from a reduced sum.  Bounds as in the tests of short lists: the norm is off
by at most 0.5 * 17 * 2^-24 + 2^-24, a clipped value by the norm's error, two roundings in fp32 and one to its type."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
NORM_TOL = 0.5 * 17 * 2.0 ** -24 + 2.0 ** -24
F, B = torch.float32, torch.bfloat16


def total(ts):
    return sum(float(p.double().square().sum()) for t in ts for p in t.split(1 << 26))


def check_values(outs, before, coef):
    for o, b in zip(outs, before):
        tol = (NORM_TOL + 2 * 2.0 ** -24 + HALF[o.dtype]) * (1 + 2.0 ** -7)
        for x, y in zip(o.split(1 << 26), b.split(1 << 26)):
            want = y.double() * coef
            assert bool(((x.double() - want).abs() <= tol * want.abs()).all())


LISTS = {"one": [(6_000_001, F)], "one in bf16": [(20_000_003, B)], "mixed": [(3_000_001, F), (17, B), (0, F), (5_000_000, B), (1, F), (1_000_003, F), (70_001, B)],
         "many": [(20_011 + i, F if i % 2 else B) for i in range(600)], "ends of tiles": [(8192 * 300, F), (16384 * 300 + 1, B), (8192 * 300 - 1, F)],
         "nine tiles a CTA": [(2 ** 29 + 100_003, F)]}


@pytest.mark.parametrize("name", LISTS)
def test_every_value(lgn, name):
    g = torch.Generator(device="cuda").manual_seed(len(name))
    before = [torch.randn(n, generator=g, device="cuda").to(dt) for n, dt in LISTS[name]]
    sq = total(before)
    norm = math.sqrt(sq)
    rec, ws = lgn.new_norm_record("cuda"), lgn.new_clip_workspace("cuda", len(before))
    ws.fill_(0xEE)
    lgn.lgn_grad_norm(lgn.make_grads(before), rec, ws)
    r = lgn.read_norm_record(rec)
    assert abs(r["norm"] - norm) <= NORM_TOL * norm and r["n_nonfinite"] == 0 and r["coef"] == 1.0
    coef = 1 / 3
    place = [t.clone() for t in before]
    lgn.lgn_clip_grad_norm(lgn.make_grads(place), norm / 3, rec, ws)
    assert lgn.read_norm_record(rec)["norm"] == r["norm"]
    check_values(place, before, coef)
    for shift in (0, 3):
        bufs = [torch.full((t.numel() + 8,), 9.0, dtype=t.dtype, device="cuda") for t in before]
        outs = [b[shift:shift + t.numel()] for b, t in zip(bufs, before)]
        lgn.lgn_clip_grad_norm(lgn.make_grads(before, outs), norm / 3, rec, ws)
        for o, p, b in zip(outs, place, bufs):
            assert torch.equal(o, p) and bool((b[:shift] == 9.0).all()) and bool((b[shift + o.numel():] == 9.0).all())
    del place
    lgn.sum_sq_of(rec).fill_(4 * sq)                               # another rank's share of the same list
    lgn.lgn_clip_apply(lgn.make_grads(before, outs), norm, rec)
    check_values(outs, before, 0.5)
