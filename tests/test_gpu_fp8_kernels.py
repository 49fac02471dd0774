"""Every kernel of the 8-bit product, each by a size that the choice sends to it (the log says which ran): plain and accumulating, both
formats, outputs of whole and of odd rows, contractions of several chunks, against fp64.

Bound: as for the product's other tests, (G + 32) 2^-23 sum |a b| with G = ceil(k / 32), half a unit of the output's type, and when
accumulating half a unit more for the old value."""
import os
import re
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROWS, SWAP, SPLIT = 0, 1, 2
# kernel: CTAs per tile, tile rows, tile columns, form, output -> sizes (m, n, k, elements added to the output's rows)
KERNELS = {
    ("single", 128, 64, SWAP, "f32"): [(64, 1000, 520, 0), (1, 3, 260, 1)],
    ("single", 128, 64, SWAP, "bf16"): [(64, 1000, 520, 0), (1, 3, 260, 1)],
    ("single", 128, 64, SPLIT, "f32"): [(4, 512, 4096, 0), (4, 40, 1300, 3), (130, 520, 5000, 1)],
    ("single", 128, 64, SPLIT, "bf16"): [(4, 512, 4096, 0), (4, 40, 1300, 3), (130, 520, 5000, 1)],
    ("single", 128, 128, ROWS, "f32"): [(777, 2504, 1000, 0), (1920, 2052, 520, 4)],
    ("single", 128, 128, ROWS, "bf16"): [(777, 2504, 1000, 0), (1152, 2048, 1000, 8)],
    ("single", 128, 128, SWAP, "f32"): [(2880, 3001, 520, 0), (3000, 3001, 520, 2)],
    ("single", 128, 128, SWAP, "bf16"): [(960, 1201, 1000, 0), (520, 2052, 1000, 1)],
    ("pairs", 256, 128, ROWS, "f32"): [(2048, 2304, 1300, 0), (2050, 520, 1000, 4)],
    ("pairs", 256, 128, ROWS, "bf16"): [(2050, 2504, 1300, 0), (1920, 520, 1300, 8)],
    ("pairs", 256, 128, SWAP, "f32"): [(960, 1201, 1000, 0), (520, 2501, 1000, 2)],
    ("pairs", 256, 128, SWAP, "bf16"): [(960, 1201, 1300, 0), (520, 2501, 1300, 2)],
    ("pairs", 256, 192, ROWS, "f32"): [(2050, 2304, 2100, 0), (4100, 520, 700, 4), (1920, 1192, 3300, 0)],
    ("pairs", 256, 192, SWAP, "f32"): [(4100, 3001, 700, 0), (1920, 1201, 2100, 1)],
    ("pairs", 256, 256, ROWS, "bf16"): [(3000, 3000, 700, 0), (4100, 3000, 2100, 8), (2880, 1200, 520, 0), (2880, 1200, 5000, 0)],
    ("pairs", 256, 256, SWAP, "bf16"): [(2880, 1201, 520, 0), (2880, 1201, 2100, 2), (2880, 1201, 640, 0)],
}


def cases():
    for i, ((ctas, rows, cols, form, od), sizes) in enumerate(KERNELS.items()):
        for j, size in enumerate(sizes):
            yield (ctas, str(rows), str(cols), str(form)), od, size, ((i + j) % 2, (i + j + 1) % 2 if j else 0)


def child():
    sys.path.insert(0, os.path.join(ROOT, "tests"))
    sys.path.insert(0, ROOT)
    from paper_2006_08173_b200 import binding as lgn
    from test_gpu_fp8 import values as inputs
    from test_gpu_fp8_sums import values
    for _, od, (m, n, k, more), (fa, fb) in cases():
        dtype, half = (torch.float32, 2.0 ** -24) if od == "f32" else (torch.bfloat16, 2.0 ** -8)
        a, _ = lgn.lgn_fp8_quantize(inputs(m, k, m + k, torch.float32), fa)
        b, _ = lgn.lgn_fp8_quantize(inputs(n, k, n + 3 * k, torch.bfloat16), fb, lgn.BLOCK_SQUARE)
        av, bv = values(a, 0, k), values(b, 0, k)
        want, mag = av @ bv.t(), av.abs() @ bv.abs().t()
        sums = ((k + 31) // 32 + 32) * 2.0 ** -23 * mag
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        buf = torch.full((m + 2, n + more), 7.0, dtype=dtype, device="cuda")
        out = buf[1:m + 1, :n]
        lgn.lgn_fp8_matmul(a, b, out=out, status=status)
        first = out.double()
        ok = bool(((first - want).abs() <= sums + half * (want.abs() + sums)).all())
        lgn.lgn_fp8_matmul(a, b, out=out, accumulate=True, status=status)
        total = want + first
        tol = sums + 2 * half * (total.abs() + sums) + 2.0 ** -23 * first.abs()
        ok2 = bool(((out.double() - total).abs() <= tol).all())
        around = bool((buf[0] == 7.0).all() and (buf[-1] == 7.0).all() and (buf[:, n:] == 7.0).all())
        print("RESULT", ok, ok2, around, int(status.item()), flush=True)


def test_every_kernel():
    r = subprocess.run([sys.executable, __file__], cwd=ROOT, env=dict(os.environ, LGN_LOG="1"), capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stderr[-3000:]
    taken = re.findall(r"fp8_matmul: m (\d+) n (\d+) k (\d+), (\w+), tile (\d+) x (\d+), form (\d)", r.stderr)
    results = re.findall(r"RESULT (.*)", r.stdout)
    listed = list(cases())
    assert len(results) == len(listed) and len(taken) == 2 * len(listed)
    for i, (kernel, od, (m, n, k, more), _) in enumerate(listed):
        for line in taken[2 * i:2 * i + 2]:
            assert line == (str(m), str(n), str(k), *kernel), (line, kernel, od)
        assert results[i] == "True True True 0", (kernel, od, (m, n, k, more), results[i])


if __name__ == "__main__":
    child()
