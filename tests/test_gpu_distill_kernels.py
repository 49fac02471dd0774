"""Every kernel of the distillation loss (the log says which ran), the one-warp kernels for many short rows in particular, against fp64.

The bounds are those of test_gpu_distill.py: 400 units of 2^-24 and 3 per unit of the exponent's argument for a softmax value.  What they have to cover:
an exponential's 4 units (base-2 approximation, 2^-22) or, where the gradient of bf16 logits takes it from a polynomial, 49 (2.9e-6); a row's sum by the
mean error of its terms, 4, and one rounding per addition of the longest chain, 64 values in a thread, 5 shuffles, 3 levels of warps and 3 of CTAs;
the quotient by the sum (1), two products and the addition of both parts (3): 49 + 4 + 75 + 1 + 3 = 132."""
import os
import re
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# (tokens, vocab, top): one warp per row from 8 rows per SM on, for rows of up to 512 pieces of 16 bytes and 128 entries
ONE_WARP = {"bf16": [(1500, 1000, 17), (2000, 4001, 128), (1200, 37, 3), (1184, 4089, 1), (1300, 500, 0), (1250, 1, 1)],
            "f32": [(1500, 1000, 17), (2000, 2001, 128), (1200, 37, 3), (1184, 2045, 1), (1300, 500, 0), (1250, 1, 1)]}
LONGER = {"bf16": [(300, 1000, 17), (1200, 1000, 129), (40, 20000, 33)], "f32": [(300, 1000, 17), (1200, 1000, 129), (40, 20000, 33)]}
WAYS = [(1.0, 1.0, False), (1.0, 0.4, True), (2.5, 0.3, True), (0.7, 1.0, True), (3.0, 0.0, True)]


def entries(ids, z, labels, v, seed):
    """Duplicate places, some of them the label's; masked teacher's logits; places outside."""
    g = torch.Generator().manual_seed(seed)
    pick = torch.randint(0, 8, (ids.shape[0],), generator=g).cuda()
    if ids.shape[1]:
        labels = torch.where(pick == 0, ids[:, 0], labels)
        ids = torch.where((pick == 1)[:, None], ids[:, :1], ids)
        ids = torch.where((pick == 2)[:, None], v, ids)
        z = torch.where((pick == 3)[:, None], -float("inf"), z)
        ids[:, ids.shape[1] // 2] = torch.where(pick == 4, ids[:, 0], ids[:, ids.shape[1] // 2])
    return ids, z, labels


def child():
    sys.path.insert(0, os.path.join(ROOT, "tests"))
    sys.path.insert(0, ROOT)
    from paper_2006_08173_b200 import binding as lgn
    from test_gpu_distill import DT, check, check_call, inputs, reference
    for dtype in ("bf16", "f32"):
        print("type", dtype, file=sys.stderr, flush=True)
        for t, v, top in ONE_WARP[dtype] + LONGER[dtype]:
            s, ids, z, labels, weight = inputs(t, v, top, t + v + top, DT[dtype])
            ids, z, labels = entries(ids, z, labels, v, top)
            for temp, alpha, labelled in WAYS:
                check_call(lgn, s, ids, z, labels if labelled else None, temp, alpha, weight)
        # rows at odd addresses, gradients over the logits or aligned differently, what lies around
        for t, v, top in ONE_WARP[dtype][:3]:
            s, ids, z, labels, weight = inputs(t, v + 9, top, v, DT[dtype])
            ids, labels = torch.where(ids >= v, -1, ids), torch.where(labels >= v, -1, labels)
            for lo in (0, 1, 3):
                view = s[:, lo:lo + v]
                loss, bound, d, dbound = reference(view, ids, z, labels, 1.3, 0.5, weight)
                for shift in (0, 1, 4):
                    whole = torch.full((t + 2, v + 11), -5.0, dtype=DT[dtype], device="cuda")
                    out = whole[1:t + 1, shift:shift + v]
                    got, _ = lgn.lgn_distill_loss(view, ids, z, labels, 1.3, 0.5, weight, dlogits=out)
                    check(got, loss, bound)
                    check(out, d, dbound)
                    out.fill_(-5.0)
                    assert (whole == -5.0).all()
                copy = s.clone()
                place = copy[:, lo:lo + v]
                lgn.lgn_distill_loss(place, ids, z, labels, 1.3, 0.5, weight, dlogits=place)
                check(place, d, dbound)
                place.copy_(view)
                assert torch.equal(copy, s)
        # values that are not finite
        s, ids, z, labels, weight = inputs(1200, 300, 6, 6, DT[dtype])
        ids[:] = torch.arange(6) * 3
        s[0, 5] = float("nan"); s[1, 7] = float("inf"); s[2] = -float("inf"); s[3, 6] = -float("inf")
        s[4] = float("nan"); ids[4], labels[4] = -1, -1
        z[5, 2] = float("nan")
        labels[0:3] = 1
        for temp in (1.0, 2.0):
            loss, grad = lgn.lgn_distill_loss(s, ids, z, labels, temp, 0.5, weight, grad=True)
            assert loss[:3].isnan().all() and grad[:3].isnan().all() and loss[3] == float("inf") and grad[3].isfinite().all()
            assert loss[4] == 0 and (grad[4] == 0).all() and loss[5].isnan() and loss[6:].isfinite().all()
            want, bound, d, dbound = reference(s[6:], ids[6:], z[6:], labels[6:], temp, 0.5, weight[6:])
            check(loss[6:], want, bound)
            check(grad[6:], d, dbound)
    print("done", file=sys.stderr)


def test_every_kernel():
    env = dict(os.environ, LGN_LOG="1")
    r = subprocess.run([sys.executable, os.path.abspath(__file__)], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and r.stderr.rstrip().endswith("done"), r.stderr[-3000:]
    ran, dtype = set(), None
    for line in r.stderr.splitlines():
        if line.startswith("type "):
            dtype = line[5:]
        m = re.match(r"\[lgn\] distill_loss: .*, (one|two) softmax(?:es)?, (\d+) threads, \d+ CTAs per row(, gradient)?", line)
        if m:
            ran.add((dtype, m.group(1), int(m.group(2)), m.group(3) is not None))
    assert ran == {(d, n, t, g) for d in ("bf16", "f32") for n in ("one", "two") for g in (False, True) for t in (32, 64, 128 if g else 256)}


if __name__ == "__main__":
    child()
