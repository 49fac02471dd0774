"""A grouped product whose first copies never come ends by itself with a status, in each of its forms, and the next one is right."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gradient,rows,n,k", [
    (False, 3, 256, 2048),              # shares of k
    (False, 200, 256, 256),             # lone CTAs
    (False, 1500, 512, 256),            # pairs
    (True, 300, 304, 304),              # lone CTAs; the groups end inside a step
    (True, 20, 128, 128),               # the first step is a group's last
    (True, 4000, 128, 128),             # rows shared out
    (True, 1500, 1024, 1024)])          # pairs
def test_time_out(lgn, gradient, rows, n, k):
    torch.manual_seed(0)
    a = torch.randn(rows, n if gradient else k, device="cuda").bfloat16()
    b = torch.randn(*((rows, k) if gradient else (2, n, k)), device="cuda").bfloat16()
    out = torch.empty(*((2, n, k) if gradient else (rows, n)), device="cuda")
    offsets = torch.tensor([0, rows // 3, rows], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lgn.lgn_selftest_grouped_wait_expires(a, b, offsets, out, status, gradient=gradient)
    torch.cuda.synchronize()
    assert int(status.item()) == 5
    status.zero_()
    if gradient:
        got = lgn.lgn_grouped_weight_grad(a, b, offsets, status=status)
        want = torch.stack([a[:rows // 3].double().t() @ b[:rows // 3].double(), a[rows // 3:].double().t() @ b[rows // 3:].double()])
    else:
        got = lgn.lgn_grouped_matmul(a, b, offsets, out_dtype=torch.float32, status=status)
        want = torch.cat([a[:rows // 3].double() @ b[0].double().t(), a[rows // 3:].double() @ b[1].double().t()])
    assert int(status.item()) == 0
    terms = rows if gradient else k
    # sums of `terms` products of normal values: (terms / 16 + 32) 2^-23 of at most 40 terms in magnitude
    assert bool(((got.double() - want).abs() <= ((terms + 15) // 16 + 32) * 2.0 ** -23 * 40.0 * terms).all())
