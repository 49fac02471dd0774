"""The limit of the product's waits does not count the time that earlier work on the stream takes: a product may become
resident beside that work, and must not give up on operands that it was not yet allowed to fetch."""
import pytest
import torch

from test_gpu_fp8 import values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k,od", [(4, 64, 256, torch.float32), (4, 512, 4096, torch.bfloat16), (960, 1201, 1000, torch.bfloat16),
                                      (2048, 2304, 512, torch.bfloat16)], ids=["lone", "shares of k", "lone 128", "pairs"])
def test_a_product_behind_work_that_takes_longer_than_the_limit(lgn, m, n, k, od):
    """The work ahead is one CTA that waits its limit out, longer than the limit of the product behind it."""
    slow_a, _ = lgn.lgn_fp8_quantize(values(4, 256, 1, torch.bfloat16), 0)
    slow_b, _ = lgn.lgn_fp8_quantize(values(64, 256, 2, torch.bfloat16), 0)
    slow_out = torch.empty(4, 64, device="cuda")
    a, _ = lgn.lgn_fp8_quantize(values(m, k, 3, torch.bfloat16), 0)
    b, _ = lgn.lgn_fp8_quantize(values(n, k, 4, torch.bfloat16), 0)
    want, out = lgn.lgn_fp8_matmul(a, b, out_dtype=od), torch.empty(m, n, dtype=od, device="cuda")
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    lgn.lgn_selftest_matmul_wait_expires(slow_a, slow_b, slow_out, status[:1])
    lgn.lgn_fp8_matmul(a, b, out=out, status=status[1:])
    torch.cuda.synchronize()
    assert status.tolist() == [5, 0]                              # LGN_ERR_TIMEOUT is the first one's own
    assert torch.equal(out, want)
