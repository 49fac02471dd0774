"""Gradients whose shared memory lies just below and above 48 KB, in a process in which no larger call has raised the kernels' limit."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# tokens, vocab, top, type: 16 (bf16 131072, fp32 32000 over 200 rows), 15 (122000) and 14 (114000) pieces per thread; dynamic sizes of 48 KB minus 112 to
# minus 0 bytes, and the first sizes on either side that need no rule of their own
SIZES = [(3, 131072, 660, "bf16"), (3, 131072, 672, "bf16"), (3, 131072, 675, "bf16"), (3, 131072, 681, "bf16"), (200, 32000, 675, "f32"), (3, 122000, 842, "bf16"), (3, 122000, 845, "bf16"),
         (3, 122000, 852, "bf16"), (2, 114000, 1015, "bf16"), (2, 114000, 1023, "bf16"), (3, 131072, 682, "bf16"), (3, 122000, 853, "bf16"), (2, 114000, 1024, "bf16")]


def child():
    sys.path.insert(0, os.path.join(ROOT, "tests"))
    sys.path.insert(0, ROOT)
    from paper_2006_08173_b200 import binding as lgn
    from test_gpu_distill import DT, check_call, inputs
    for temp in (1.0, 2.5):
        for t, v, top, dtype in SIZES:
            s, ids, z, labels, weight = inputs(t, v, top, t + v + top, DT[dtype])
            check_call(lgn, s, ids, z, labels, temp, 0.4, weight)
    print("done")


def test_below_and_above_48_kb():
    r = subprocess.run([sys.executable, os.path.abspath(__file__)], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and r.stdout.rstrip().endswith("done"), (r.stdout + r.stderr)[-3000:]


if __name__ == "__main__":
    child()
