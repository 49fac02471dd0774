"""The table gradient on long batches: windows of more than eight tokens, which only large batches take, and the sort of batches that do
not stay in registers.  Against fp64 sums on the GPU.

Bound: a sum of c rows in fp32, in any order, is off by at most (c - 1) 2^-24 sum |dout| and its scaling by 2^-24 more; an accumulating
call adds 2^-24 of the result, and the output's type rounds by half a unit."""
import os
import re
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def ids_of(n, vocab, kind, dtype):
    g = torch.Generator(device="cuda").manual_seed(n + vocab)
    r = lambda lo, hi: torch.randint(lo, hi, (n,), generator=g, device="cuda")
    if kind == "uniform":
        ids = r(0, vocab)
    elif kind == "one":                                            # one run through all windows
        ids = torch.full((n,), vocab // 3, device="cuda")
    elif kind == "skewed":                                         # runs of thousands, of several windows, of one token
        ids = (torch.rand(n, generator=g, device="cuda") ** 8 * vocab).long().clamp_(max=vocab - 1)
    else:                                                          # half left out: they end the list in the middle of a window
        ids = r(-vocab, vocab)
    return ids.to(dtype)


def check(lgn, n, vocab, dim, kind, ddt, odt, idt, pad, scale=0.75):
    g = torch.Generator(device="cuda").manual_seed(n)
    dout = torch.randn(n, dim, generator=g, device="cuda").to(DT[ddt])
    ids = ids_of(n, vocab, kind, idt)
    keep = ((ids >= 0) & (ids < vocab) & (ids != pad)).nonzero()[:, 0]
    rows = ids[keep].long()
    want, mag = (torch.zeros(vocab, dim, dtype=torch.float64, device="cuda") for _ in range(2))
    for part in torch.arange(keep.numel(), device="cuda").split(16384):
        d = dout[keep[part]].double()
        want.index_add_(0, rows[part], d)
        mag.index_add_(0, rows[part], d.abs())
    count = torch.bincount(rows, minlength=vocab).double()[:, None]
    want, mag = want * scale, mag * scale
    sums = count * 2.0 ** -24 * mag * (1 + 1e-5)
    got = lgn.lgn_embedding_grad(dout, ids, vocab, scale, padding_idx=pad, out_dtype=DT[odt])
    tol = sums + HALF[DT[odt]] * (want.abs() + sums)
    assert bool(((got.double() - want).abs() <= tol).all())
    assert bool((got[count[:, 0] == 0] == 0).all())
    assert torch.equal(got, lgn.lgn_embedding_grad(dout, ids, vocab, scale, padding_idx=pad, out_dtype=DT[odt]))
    before = torch.randn(vocab, dim, generator=g, device="cuda").to(DT[odt])
    out = before.clone()
    lgn.lgn_embedding_grad(dout, ids, vocab, scale, padding_idx=pad, out=out, accumulate=True)
    total = want + before.double()
    tol = sums + 2.0 ** -24 * (total.abs() + sums)
    tol = tol + HALF[DT[odt]] * (total.abs() + tol)
    assert bool(((out.double() - total).abs() <= tol).all())
    assert torch.equal(out[count[:, 0] == 0], before[count[:, 0] == 0])


# tokens, table rows, columns (whole, pairs, odd: three widths of access), tokens per window
WINDOWS = [(4200, 700, 4096, 16), (5000, 1003, 4096, 32), (20000, 3001, 2048, 64), (20000, 515, 2046, 64), (20000, 700, 2047, 64), (66000, 900, 2500, 128)]


@pytest.mark.parametrize("kind", ["uniform", "one", "skewed", "outside"])
@pytest.mark.parametrize("n,vocab,dim,window", WINDOWS)
def test_windows_of_more_than_eight_tokens(lgn, n, vocab, dim, window, kind):
    for i, (ddt, odt) in enumerate((("bf16", "f32"), ("f32", "bf16"))):
        check(lgn, n, vocab, dim, kind, ddt, odt, (torch.int64, torch.int32)[i], vocab // 2 if kind == "skewed" else -1)


def test_the_windows_are_what_they_are_said_to_be():
    code = """
import torch
from paper_2006_08173_b200 import binding as lgn
for n, vocab, dim, _ in {cases}:
    lgn.lgn_embedding_grad(torch.zeros(n, dim, device="cuda"), torch.zeros(n, dtype=torch.int64, device="cuda"), vocab)
torch.cuda.synchronize()
"""
    r = subprocess.run([sys.executable, "-c", code.format(cases=WINDOWS)], cwd=ROOT, env=dict(os.environ, LGN_LOG="1"), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    windows = [int(w) for w in re.findall(r"embedding_grad: .* (\d+) windows", r.stderr)]
    assert windows == [-(-n // w) for n, _, _, w in WINDOWS]


@pytest.mark.parametrize("kind", ["uniform", "skewed", "outside"])
@pytest.mark.parametrize("n,vocab,dim", [(131072, 70001, 8), (131073, 70001, 8), (140001, 515, 12), (300000, 600011, 3), (1000003, 30, 4)])
def test_sorts_of_more_tokens_than_registers_hold(lgn, n, vocab, dim, kind):
    """From 131073 tokens up a warp's share of the list is read again in every pass."""
    check(lgn, n, vocab, dim, kind, "f32", "f32", torch.int64, 2)
