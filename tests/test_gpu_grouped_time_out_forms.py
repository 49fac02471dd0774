"""Bounded waits of the grouped products, form by form: the log says which kernel ran, every CTA's first copy is withheld, the kernel ends by itself
with a status, and the same product done properly afterwards keeps the bounds of test_gpu_grouped.py and test_gpu_int8.py."""
import os
import re
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROWS, SWAP, GRAD, SHARE, TURN = 0, 1, 2, 3, 4
# gradient (2: 8-bit integers), group ends, n, k, output -> form, tile, shares
CASES = [
    (False, [0, 1000, 2443], 1744, 264, "f32", ROWS, "256 x 256", 1),
    (False, [0, 1000, 2443], 1744, 264, "bf16", ROWS, "256 x 256", 1),
    (False, [0, 700, 1500], 512, 256, "f32", ROWS, "128 x 128", 1),
    (False, [0, 200, 200, 500, 835], 2328, 1016, "f32", TURN, "256 x 256", 1),
    (False, [0, 3, 17, 17, 30], 360, 1616, "f32", SWAP, "32 x 128", 8),
    (False, [0, 158, 258], 328, 760, "f32", SWAP, "32 x 128", 4),
    (False, [0, 50, 100, 150], 1784, 2336, "f32", SWAP, "64 x 128", 4),
    (True, [0, 100, 300], 304, 304, "f32", GRAD, "128 x 128", 1),              # groups end inside a step
    (True, [0, 6, 20], 128, 128, "bf16", GRAD, "128 x 128", 1),                # the first step is a group's last
    (True, [0, 300, 607], 1688, 1168, "f32", GRAD, "256 x 256", 1),            # pairs: both CTAs clear rows of a last step
    (True, [0, 5, 607], 1688, 1168, "f32", GRAD, "256 x 256", 1),              # pairs whose first step is a group's last
    (True, [0, 5, 607], 1688, 1168, "bf16", GRAD, "256 x 256", 1),
    (True, [0, 320, 640], 2048, 2304, "f32", GRAD, "256 x 256", 1),            # pairs, nothing to clear
    (True, [0, 1900, 3802], 864, 328, "f32", SHARE, "128 x 128", 2),
    (True, [0, 3240], 744, 696, "f32", SHARE, "128 x 128", 4),
    (True, [0, 1300, 2837], 672, 112, "f32", SHARE, "128 x 128", 8),
    (2, [0, 1, 3, 3, 3, 4, 5, 6, 7, 8, 10, 12], 760, 728, "f32", TURN, "256 x 256", 1),
    (2, [0, 4912], 712, 1704, "f32", ROWS, "256 x 256", 1),
    (2, [0, 118], 1584, 1000, "f32", ROWS, "256 x 128", 1),
    (2, [0, 60, 160], 1408, 824, "bf16", ROWS, "256 x 128", 1),
    (2, [0, 113], 1992, 112, "f32", ROWS, "128 x 128", 1),
    (2, [0, 5, 5, 15], 1184, 2736, "f32", SWAP, "32 x 128", 8),
]


def child():
    sys.path.insert(0, os.path.join(ROOT, "tests"))
    sys.path.insert(0, ROOT)
    from paper_2006_08173_b200 import binding as lgn
    from test_gpu_grouped import check, forward, gradient as grad, values
    import test_gpu_int8 as int8
    for i, (gradient, ends, n, k, od, *_) in enumerate(CASES):
        rows, groups, dtype = ends[-1], len(ends) - 1, torch.bfloat16 if od == "bf16" else torch.float32
        if gradient == 2:
            a, b = lgn.lgn_int8_quantize(int8.values(rows, k, i)), lgn.lgn_int8_quantize(int8.values(groups * n, k, i + 50))
        else:
            a = values(rows, n if gradient else k, seed=i)
            b = values(*((rows, k) if gradient else (groups, n, k)), seed=i + 50)
        out = torch.empty(*((groups, n, k) if gradient == 1 else (rows, n)), dtype=dtype, device="cuda")
        offsets = torch.tensor(ends, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        print("case", i, file=sys.stderr, flush=True)
        lgn.lgn_selftest_grouped_wait_expires(a, b, offsets, out, status, gradient=gradient == 1)
        torch.cuda.synchronize()
        assert int(status.item()) == 5, i
        status.zero_()
        if gradient == 2:
            full = int8.product(a, b, dtype)
            want = torch.cat([full[ends[e]:ends[e + 1], e * n:(e + 1) * n] for e in range(groups)])
            int8.check(lgn.lgn_int8_matmul(a, b, out_dtype=dtype, offsets=offsets, status=status), want)
        elif gradient:
            check(lgn.lgn_grouped_weight_grad(a, b, offsets, out_dtype=dtype, status=status), *grad(a, b, ends), rows)
        else:
            check(lgn.lgn_grouped_matmul(a, b, offsets, out_dtype=dtype, status=status), *forward(a, b, ends, False), k)
        assert int(status.item()) == 0, i
    print("done", file=sys.stderr)


def test_every_form_ends():
    env = dict(os.environ, LGN_LOG="1")
    r = subprocess.run([sys.executable, os.path.abspath(__file__)], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and r.stderr.rstrip().endswith("done"), r.stderr[-3000:]
    ran, case = {}, None
    for line in r.stderr.splitlines():
        if line.startswith("case "):
            case = int(line[5:])
        m = re.match(r"\[lgn\] grouped: .*, tile (\d+ x \d+), form (\d), split (\d)", line)
        if m:
            ran.setdefault(case, []).append((int(m.group(2)), m.group(1), int(m.group(3))))
    for i, (*_, form, tile, split) in enumerate(CASES):
        assert len(ran[i]) == 2 and ran[i][0] == ran[i][1], (i, ran[i])
        assert ran[i][0][:2] == (form, tile) and ran[i][0][2] == split, (i, ran[i])


if __name__ == "__main__":
    child()
