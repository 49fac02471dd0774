"""A weight gradient in which one group keeps a CTA busy for longer than the kernel's bounded waits last."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_group_that_takes_seconds(lgn):
    """160 groups, all rows but a few in the last but one, whose end lies inside a step of the contraction: the warp that clears the rows behind it has
    nothing to do for all of that time.

    Operands are powers of two, so sums of 512 products and their sums are exact; the last one, of less than 512, is rounded to fp32."""
    rows, groups, m, n = 1 << 29, 160, 8, 8
    up, down = (2.0 ** (s * torch.arange(8.0, device="cuda")) for s in (1, -1))
    dy, x = (torch.empty(rows, 8, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dy[:], x[:] = up.bfloat16(), down.bfloat16()
    end = rows - 5
    x[end:] = float("nan")
    offsets = torch.full((groups + 1,), end, device="cuda")
    offsets[:groups - 1] = 0
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = lgn.lgn_grouped_weight_grad(dy, x, offsets, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    want = float(end) * up.double()[:, None] * down.double()[None, :]
    assert bool(((out[groups - 2].double() - want).abs() <= 2.0 ** -24 * want).all())
    assert not out[:groups - 2].any() and not out[groups - 1].any()
    del dy, x
    torch.cuda.empty_cache()
