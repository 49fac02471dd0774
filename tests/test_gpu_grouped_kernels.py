"""Every kernel of the grouped products, each by a size that the choice sends to it (the log says which ran), against fp64, with the
bounds of test_gpu_grouped.py and test_gpu_int8.py."""
import os
import re
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROWS, SWAP, GRAD, SHARE, TURN = 0, 1, 2, 3, 4
# product, form, tile, output -> sizes (rows, groups, n, k) (gradient: m = n, n = k)
KERNELS = {
    ("X W^T", ROWS, "256 x 256", "bf16"): [(3484, 18, 1040, 512), (13409, 3, 536, 1344)],
    ("X W^T", ROWS, "128 x 128", "bf16"): [(3504, 7, 192, 240), (7118, 10, 240, 576)],
    ("X W^T", SWAP, "32 x 128", "bf16"): [(63, 5, 472, 2336), (620, 40, 104, 3344)],
    ("X W^T", SWAP, "64 x 128", "bf16"): [(3644, 17, 184, 1872), (5806, 14, 96, 3288)],
    ("X W^T", TURN, "256 x 256", "bf16"): [(103, 11, 328, 1272), (9609, 57, 168, 832)],
    ("X W^T", ROWS, "256 x 256", "f32"): [(7081, 2, 1840, 96), (10509, 2, 144, 2344)],
    ("X W^T", ROWS, "128 x 128", "f32"): [(2988, 2, 464, 384), (8023, 2, 256, 720)],
    ("X W^T", SWAP, "32 x 128", "f32"): [(2304, 3, 208, 1896), (114, 59, 800, 376)],
    ("X W^T", SWAP, "64 x 128", "f32"): [(1947, 11, 328, 1640), (1433, 38, 1744, 248)],
    ("X W^T", TURN, "256 x 256", "f32"): [(24, 21, 208, 680), (22, 21, 544, 1248)],
    ("X W", ROWS, "256 x 256", "bf16"): [(15523, 4, 752, 152), (10254, 5, 136, 2320)],
    ("X W", ROWS, "128 x 128", "bf16"): [(119, 4, 2344, 160), (9440, 49, 104, 368)],
    ("X W", SWAP, "32 x 128", "bf16"): [(976, 52, 264, 352), (51, 4, 1856, 2136)],
    ("X W", SWAP, "64 x 128", "bf16"): [(2365, 21, 104, 3184), (9297, 3, 120, 2280)],
    ("X W", TURN, "256 x 256", "bf16"): [(27, 8, 984, 616), (3229, 49, 680, 384)],
    ("X W", ROWS, "256 x 256", "f32"): [(26826, 6, 328, 176), (18912, 7, 248, 1032)],
    ("X W", ROWS, "128 x 128", "f32"): [(11278, 11, 112, 120), (4849, 6, 888, 352)],
    ("X W", SWAP, "32 x 128", "f32"): [(197, 6, 432, 2288), (219, 35, 2008, 248)],
    ("X W", SWAP, "64 x 128", "f32"): [(211, 2, 1784, 2336), (1488, 21, 224, 3096)],
    ("X W", TURN, "256 x 256", "f32"): [(492, 5, 2192, 152), (777, 8, 3488, 376)],
    ("dY^T X", GRAD, "256 x 256", "bf16"): [(1783, 19, 488, 1616), (6344, 11, 480, 2360)],
    ("dY^T X", GRAD, "128 x 128", "bf16"): [(10, 7, 2856, 168), (180, 5, 784, 2880)],
    ("dY^T X", SHARE, "128 x 128", "bf16"): [(7266, 4, 760, 128), (27804, 4, 384, 128)],
    ("dY^T X", GRAD, "256 x 256", "f32"): [(7112, 2, 552, 1904), (16203, 5, 1448, 296)],
    ("dY^T X", GRAD, "128 x 128", "f32"): [(273, 8, 592, 688), (25, 15, 440, 1928)],
    ("dY^T X", SHARE, "128 x 128", "f32"): [(10023, 3, 496, 200), (19581, 5, 320, 448)],
    ("8-bit X W^T", TURN, "256 x 256", "bf16"): [(8, 1, 1576, 1680), (17, 9, 1856, 656)],
    ("8-bit X W^T", ROWS, "256 x 256", "bf16"): [(17018, 5, 648, 104), (21838, 15, 472, 504)],
    ("8-bit X W^T", ROWS, "256 x 128", "bf16"): [(160, 2, 1408, 824), (1069, 1, 1600, 2600)],
    ("8-bit X W^T", ROWS, "128 x 128", "bf16"): [(541, 6, 216, 264), (2208, 24, 184, 288)],
    ("8-bit X W^T", SWAP, "32 x 128", "bf16"): [(96, 2, 344, 4064), (87, 22, 816, 504)],
    ("8-bit X W^T", TURN, "256 x 256", "f32"): [(6, 1, 1488, 656), (12, 11, 760, 728)],
    ("8-bit X W^T", ROWS, "256 x 256", "f32"): [(4912, 1, 712, 1704), (10738, 1, 1648, 568)],
    ("8-bit X W^T", ROWS, "256 x 128", "f32"): [(118, 1, 1584, 1000), (10697, 1, 360, 216)],
    ("8-bit X W^T", ROWS, "128 x 128", "f32"): [(113, 1, 1992, 112), (3543, 1, 528, 104)],
    ("8-bit X W^T", SWAP, "32 x 128", "f32"): [(20, 6, 3936, 144), (15, 3, 1184, 2736)],
}


def child():
    sys.path.insert(0, os.path.join(ROOT, "tests"))
    sys.path.insert(0, ROOT)
    from paper_2006_08173_b200 import binding as lgn
    from test_gpu_grouped import check, forward, gradient, spans, values
    import test_gpu_int8 as int8
    for i, ((what, form, tile, od), sizes) in enumerate(KERNELS.items()):
        dtype = torch.bfloat16 if od == "bf16" else torch.float32
        for rows, groups, n, k in sizes:
            ends = spans(rows, groups, i + 1) if groups > 1 else [0, rows]
            offsets = torch.tensor(ends, device="cuda")
            torch.cuda.synchronize()
            print("case", what, form, tile, od, file=sys.stderr, flush=True)
            if what.startswith("8"):
                a, b = lgn.lgn_int8_quantize(int8.values(rows, k, i)), lgn.lgn_int8_quantize(int8.values(groups * n, k, i + 50))
                out = lgn.lgn_int8_matmul(a, b, out_dtype=dtype, offsets=offsets if groups > 1 else None)
                full = int8.product(a, b, dtype)
                want = torch.cat([full[ends[e]:ends[e + 1], e * n:(e + 1) * n] for e in range(groups)])
                int8.check(out, want)
            elif what == "dY^T X":
                dy, x = values(rows, n, seed=i), values(rows, k, seed=i + 50)
                check(lgn.lgn_grouped_weight_grad(dy, x, offsets, out_dtype=dtype), *gradient(dy, x, ends), rows)
            else:
                turned = what == "X W"
                x, w = values(rows, k, seed=i), values(groups, *((k, n) if turned else (n, k)), seed=i + 50)
                check(lgn.lgn_grouped_matmul(x, w, offsets, out_dtype=dtype, transposed=turned), *forward(x, w, ends, turned), k)
    print("done", file=sys.stderr)


def test_every_kernel():
    env = dict(os.environ, LGN_LOG="1")
    r = subprocess.run([sys.executable, os.path.abspath(__file__)], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and r.stderr.rstrip().endswith("done"), r.stderr[-3000:]
    ran, expect = set(), None
    for line in r.stderr.splitlines():
        if line.startswith("case "):
            expect = line[5:]
        m = re.match(r"\[lgn\] grouped: (.*), rows .*, tile (\d+ x \d+), form (\d), split", line)
        if m:
            what, tile, form = m.groups()
            assert expect in (f"{what} {form} {tile} bf16", f"{what} {form} {tile} f32"), (expect, line)
            ran.add(expect)
    assert ran == {" ".join(map(str, key)) for key in KERNELS}


if __name__ == "__main__":
    child()
