"""8-bit operands without a column, and products over them: zeros, whatever the scales' memory held before."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ends", [None, [0, 3, 3, 9], [2, 5, 7]])
@pytest.mark.parametrize("rows,n", [(9, 7), (9, 300), (500, 40), (700, 1000)])
def test_product_over_nothing(lgn, rows, n, ends, dtype):
    groups = 1 if ends is None else len(ends) - 1
    a, b = lgn.new_int8_operand(rows, 0, "cuda"), lgn.new_int8_operand(groups * n, 0, "cuda")
    a.scales.fill_(float("nan"))
    b.scales.fill_(float("inf"))
    offsets = None if ends is None else torch.tensor(ends, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = lgn.lgn_int8_matmul(a, b, out_dtype=dtype, offsets=offsets, status=status)
    assert out.shape == (rows, n) and (out == 0).all()
    out = torch.full((rows, n), 3.0, dtype=dtype, device="cuda")
    lgn.lgn_int8_matmul(a, b, out=out, offsets=offsets, status=status)
    first, last = (0, rows) if ends is None else (ends[0], ends[-1])
    assert (out[first:last] == 0).all() and (out[:first] == 3.0).all() and (out[last:] == 3.0).all() and int(status.item()) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 5, 700])
def test_scales_of_rows_without_a_column(lgn, rows, dtype):
    """The largest magnitude counts as 2^-110."""
    out = lgn.new_int8_operand(rows, 0, "cuda")
    out.scales.fill_(float("nan"))
    lgn.lgn_int8_quantize(torch.empty(rows, 0, dtype=dtype, device="cuda"), out=out)
    want = (torch.tensor(2.0 ** -110, dtype=torch.float64) / 127.0).float()
    assert torch.equal(out.scales.cpu(), want.expand(rows))
