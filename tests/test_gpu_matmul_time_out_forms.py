"""Every form of the product ends by itself when its copies do not come: lone CTAs, pairs (one and two accumulator halves per tile),
rows along either dimension of the output, tiles of several chunks of k and several tiles per CTA.  The child's log says which kernel
each size took."""
import os
import re
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# (m, n, k, output) -> CTAs per tile, tile rows, tile columns, form (0: rows, 1: swapped)
CASES = [((1920, 520, 700, "f32"), ("single", 128, 128, 0)), ((960, 1201, 1000, "bf16"), ("single", 128, 128, 1)),
         ((2048, 2304, 4096, "f32"), ("pairs", 256, 128, 0)), ((960, 1201, 1300, "bf16"), ("pairs", 256, 128, 1)),
         ((1920, 1192, 2100, "f32"), ("pairs", 256, 192, 0)), ((1920, 1201, 700, "f32"), ("pairs", 256, 192, 1)),
         ((4100, 3000, 4096, "bf16"), ("pairs", 256, 256, 0)), ((2880, 1201, 520, "bf16"), ("pairs", 256, 256, 1))]
CODE = """
import sys, time, torch
sys.path.insert(0, "tests")
from paper_2006_08173_b200 import binding as lgn
from test_gpu_fp8 import values
for m, n, k, od in {cases}:
    a, _ = lgn.lgn_fp8_quantize(values(m, k, 1, torch.bfloat16), 0)
    b, _ = lgn.lgn_fp8_quantize(values(n, k, 2, torch.bfloat16), 0)
    dt = dict(f32=torch.float32, bf16=torch.bfloat16)[od]
    want, out = lgn.lgn_fp8_matmul(a, b, out_dtype=dt), torch.empty(m, n, dtype=dt, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    t0 = time.monotonic()
    lgn.lgn_selftest_matmul_wait_expires(a, b, out, status)
    torch.cuda.synchronize()
    took, code = time.monotonic() - t0, int(status.item())
    status.zero_()
    lgn.lgn_fp8_matmul(a, b, out=out, status=status)
    print("RESULT", code, 0.5 < took < 30.0, int(status.item()), torch.equal(out, want), flush=True)
"""


def test_every_form_ends_by_itself():
    env = dict(os.environ, LGN_LOG="1")
    r = subprocess.run([sys.executable, "-c", CODE.format(cases=[c for c, _ in CASES])], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    lines = re.findall(r"fp8_matmul: m (\d+) n (\d+) k (\d+), (\w+), tile (\d+) x (\d+), form (\d)", r.stderr)
    assert len(lines) == 3 * len(CASES)
    for i, ((m, n, k, _), (ctas, rows, cols, form)) in enumerate(CASES):
        for line in lines[3 * i:3 * i + 3]:
            assert line == (str(m), str(n), str(k), ctas, str(rows), str(cols), str(form))
    assert re.findall(r"RESULT (.*)", r.stdout) == ["5 True 0 True"] * len(CASES)        # LGN_ERR_TIMEOUT, then a good product
