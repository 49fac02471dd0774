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
    ("X W^T", ROWS, "256 x 256", "bf16"): [(24359, 19, 680, 272), (14719, 3, 1296, 824)],
    ("X W^T", ROWS, "128 x 128", "bf16"): [(744, 35, 240, 264), (10818, 4, 840, 128)],
    ("X W^T", SWAP, "32 x 128", "bf16"): [(380, 12, 2016, 264), (83, 6, 744, 3512)],
    ("X W^T", SWAP, "64 x 128", "bf16"): [(687, 6, 600, 2984), (866, 36, 168, 3448)],
    ("X W^T", TURN, "256 x 256", "bf16"): [(11638, 19, 240, 184), (2784, 3, 1216, 2208)],
    ("X W^T", ROWS, "256 x 256", "f32"): [(6632, 8, 2000, 520), (14239, 10, 1944, 152)],
    ("X W^T", ROWS, "128 x 128", "f32"): [(1350, 16, 208, 168), (8, 3, 2864, 312)],
    ("X W^T", SWAP, "32 x 128", "f32"): [(103, 8, 344, 1360), (45, 3, 1616, 2240)],
    ("X W^T", SWAP, "64 x 128", "f32"): [(18900, 5, 112, 448), (29858, 57, 344, 176)],
    ("X W^T", TURN, "256 x 256", "f32"): [(19856, 33, 208, 496), (19840, 2, 136, 1344)],
    ("X W", ROWS, "256 x 256", "bf16"): [(19738, 5, 872, 360), (9695, 5, 232, 2984)],
    ("X W", ROWS, "128 x 128", "bf16"): [(52, 41, 624, 104), (5804, 14, 152, 1224)],
    ("X W", SWAP, "32 x 128", "bf16"): [(7, 2, 1464, 2288), (483, 32, 120, 3568)],
    ("X W", SWAP, "64 x 128", "bf16"): [(3381, 13, 104, 2704), (388, 5, 3720, 1048)],
    ("X W", TURN, "256 x 256", "bf16"): [(1674, 10, 1504, 232), (476, 13, 832, 1560)],
    ("X W", ROWS, "256 x 256", "f32"): [(4864, 5, 3672, 160), (11685, 2, 2592, 96)],
    ("X W", ROWS, "128 x 128", "f32"): [(4215, 3, 136, 128), (2473, 2, 752, 248)],
    ("X W", SWAP, "32 x 128", "f32"): [(11, 3, 616, 2128), (22, 10, 368, 3064)],
    ("X W", SWAP, "64 x 128", "f32"): [(18033, 49, 352, 128), (322, 16, 2840, 408)],
    ("X W", TURN, "256 x 256", "f32"): [(1190, 2, 2528, 2232), (2003, 8, 936, 2864)],
    ("dY^T X", GRAD, "256 x 256", "bf16"): [(2433, 15, 2272, 152), (23359, 13, 184, 824)],
    ("dY^T X", GRAD, "128 x 128", "bf16"): [(144, 40, 440, 216), (1106, 32, 2744, 120)],
    ("dY^T X", SHARE, "128 x 128", "bf16"): [(15769, 8, 168, 232), (7355, 3, 120, 1840)],
    ("dY^T X", GRAD, "256 x 256", "f32"): [(2695, 7, 648, 1672), (5168, 21, 1704, 472)],
    ("dY^T X", GRAD, "128 x 128", "f32"): [(107, 2, 3544, 496), (198, 31, 2792, 160)],
    ("dY^T X", SHARE, "128 x 128", "f32"): [(14441, 2, 192, 344), (21704, 2, 256, 584)],
    ("8-bit X W^T", TURN, "256 x 256", "bf16"): [(14053, 1, 168, 120), (3, 1, 3672, 3160)],
    ("8-bit X W^T", ROWS, "256 x 256", "bf16"): [(4357, 1, 3520, 1464), (10631, 4, 2240, 568)],
    ("8-bit X W^T", ROWS, "256 x 128", "bf16"): [(669, 1, 1208, 2024), (1472, 4, 808, 2376)],
    ("8-bit X W^T", ROWS, "128 x 128", "bf16"): [(3, 1, 3248, 304), (1423, 3, 2584, 184)],
    ("8-bit X W^T", SWAP, "32 x 128", "bf16"): [(122, 1, 1040, 3888), (43, 16, 2032, 440)],
    ("8-bit X W^T", SWAP, "64 x 128", "bf16"): [(484, 60, 3344, 120), (427, 35, 2736, 368)],
    ("8-bit X W^T", TURN, "256 x 256", "f32"): [(11736, 1, 248, 1312), (2884, 2, 2328, 3072)],
    ("8-bit X W^T", ROWS, "256 x 256", "f32"): [(10012, 3, 1032, 1288), (10766, 1, 2776, 320)],
    ("8-bit X W^T", ROWS, "256 x 128", "f32"): [(49, 2, 2616, 160), (1563, 1, 3320, 232)],
    ("8-bit X W^T", ROWS, "128 x 128", "f32"): [(153, 22, 736, 200), (2672, 50, 168, 536)],
    ("8-bit X W^T", SWAP, "32 x 128", "f32"): [(56, 1, 1136, 2224), (138, 7, 408, 2544)],
    ("8-bit X W^T", SWAP, "64 x 128", "f32"): [(372, 1, 2120, 3896), (3273, 20, 952, 792)],
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
