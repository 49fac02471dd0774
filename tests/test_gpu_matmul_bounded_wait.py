"""The product's device-side waits are bounded: with the first copy of every CTA withheld, the waits run out, the
kernel ends by itself and reports LGN_ERR_TIMEOUT, and the next product is right (tensor memory was given back)."""
import time

import pytest
import torch

from fp8_helpers import operand_values
from test_gpu_fp8 import check_product, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(4, 64, 256), (4, 512, 4096), (1024, 1024, 1536)],
                         ids=["lone", "shares of k", "pairs"])
def test_a_withheld_copy_ends_in_a_time_out(lgn, m, n, k):
    a, _ = lgn.lgn_fp8_quantize(values(m, k, 1, torch.bfloat16), 0)
    b, _ = lgn.lgn_fp8_quantize(values(n, k, 2, torch.bfloat16), 0)
    out = torch.empty(m, n, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    t0 = time.monotonic()
    lgn.lgn_selftest_matmul_wait_expires(a, b, out, status)
    torch.cuda.synchronize()
    took = time.monotonic() - t0
    assert int(status.item()) == 5                                # LGN_ERR_TIMEOUT
    assert 0.5 < took < 20.0
    status.zero_()
    lgn.lgn_fp8_matmul(a, b, out=out, status=status)
    assert int(status.item()) == 0
    check_product(out, operand_values(a)[0], operand_values(b)[0], k)


def test_the_self_test_refuses_bad_arguments(lgn):
    a, _ = lgn.lgn_fp8_quantize(torch.ones(4, 64, device="cuda"), 0)
    out, status = torch.empty(4, 4, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        lgn.lgn_selftest_matmul_wait_expires(lgn.lgn_fp8_quantize(torch.ones(4, 64, device="cuda"), 1)[0], a, out, status)
    raw = lgn.raw()
    assert raw.lgn_selftest_matmul_wait_expires(a._codes_ptr, a._scales_ptr, a._codes_ptr, a._scales_ptr, 4, 4, 64, out.data_ptr(), 0, None, None) == 1
    assert raw.lgn_selftest_matmul_wait_expires(a._codes_ptr, a._scales_ptr, a._codes_ptr, a._scales_ptr, 4, 4, 0, out.data_ptr(), 0, status.data_ptr(), None) == 1
