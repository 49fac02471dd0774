"""The quantiser to 8-bit integers and the product of its operands against plain fp64 forms.

Quantiser: every code and every scale exactly.  Product: the integer sum is exact; fp32 rounds it, its product
with one scale and that with the other (3 2^-24), bf16 outputs once more (2^-8)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def values(rows, cols, seed, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    x = torch.exp(2.0 * torch.randn(rows, cols, generator=g) - 3.0) * torch.where(torch.rand(rows, cols, generator=g) < 0.5, -1.0, 1.0)
    x[torch.rand(rows, cols, generator=g) < 0.2] = 0.0
    return x.to(dtype).cuda()


def reference(x):
    """(codes, scales) in fp64, from the definition: the quotients rounded to fp32, the product rounded to even."""
    x = x.double().cpu()
    a = x.abs().amax(dim=1) if x.shape[1] else torch.zeros(x.shape[0], dtype=torch.float64)
    a = torch.clamp(a, min=2.0 ** -110)
    seven = torch.full_like(a, 127.0)
    per, scale = (seven / a).float().double(), (a / seven).float()
    return torch.round(x * per[:, None]), scale


def check_operand(op, x):
    want, scale = reference(x)
    rows, k = x.shape
    codes = op.codes.view(rows, -1).cpu()
    finite = torch.isfinite(x.double().cpu()).all(dim=1)
    assert torch.equal(codes[finite, :k].double(), want[finite])
    assert torch.equal(op.scales.cpu()[finite], scale[finite])
    assert op.scales.cpu()[~finite].isnan().all()
    assert not codes[:, k:].any()


SIZES = [(1, 1), (1, 4096), (3, 17), (4, 256), (5, 257), (9, 1024), (700, 1000), (600, 2048), (601, 2049), (127, 8192), (2, 16384), (3, 20001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantiser(lgn, rows, cols, dtype):
    x = values(rows, cols, rows + 3 * cols, DT[dtype])
    check_operand(lgn.lgn_int8_quantize(x), x)


def test_quantiser_views_and_out(lgn):
    big = values(70, 1000, 3, torch.bfloat16)
    for view in (big[:, :640], big[3:, 1:700], big[::2, 8:136], big[5:6, 3:9]):
        out = lgn.new_int8_operand(*view.shape, "cuda")
        out.codes.fill_(77)
        assert lgn.lgn_int8_quantize(view, out=out) is out
        check_operand(out, view)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantiser_extremes(lgn, dtype):
    """Ties, zeros, subnormals, the largest floats, a row's maximum at every place of a warp and CTA, infinities and NaN."""
    x = torch.zeros(300, 300)
    x[0, :] = torch.arange(300) - 150.0
    x[1, :255] = (torch.arange(255) - 127) / 2.0; x[1, 299] = 127.0          # halves: ties
    x[2, 7] = torch.finfo(torch.float32).max / 2
    x[3, :] = 1e-45
    x[4, 0] = 2.0 ** -110; x[4, 1] = -(2.0 ** -111)
    x[5, 3] = float("inf"); x[6, 3] = float("-inf"); x[7, 299] = float("nan")
    x[8, :] = -0.0
    for i in range(9, 300):
        x[i, i] = -float(i)
        x[i, (i * 7) % 300] += 0.5 * i
    x = x.to(DT[dtype]).cuda()
    check_operand(lgn.lgn_int8_quantize(x), x)


def product(a, b, dtype):
    return (a.codes.view(a.rows, -1).double() @ b.codes.view(b.rows, -1).double().t()) * a.scales.double()[:, None] * b.scales.double()


def check(out, want):
    tol = want.abs() * (3.001 * 2.0 ** -24 + (2.0 ** -8 * 1.001 if out.dtype == torch.bfloat16 else 0.0))
    bad = ~((out.double() - want).abs() <= tol) & ~(out.isnan() & want.isnan())
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4], out[bad][:4], want[bad][:4])


PRODUCTS = [(1, 1, 1), (1, 128, 128), (4, 4096, 512), (5, 333, 1000), (33, 64, 4096), (64, 1000, 2048), (128, 128, 32), (128, 256, 128), (130, 200, 300),
            (257, 513, 640), (777, 2505, 1003), (300, 1, 77), (1000, 40, 1536), (2048, 2048, 256), (3000, 2501, 700), (2049, 4112, 1300), (16, 24, 131072)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(lgn, m, n, k, dtype):
    a, b = lgn.lgn_int8_quantize(values(m, k, m + k)), lgn.lgn_int8_quantize(values(n, k, n + 3 * k, torch.bfloat16))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = lgn.lgn_int8_matmul(a, b, out_dtype=DT[dtype], status=status)
    assert int(status.item()) == 0
    check(out, product(a, b, DT[dtype]))


def test_largest_sums(lgn):
    """Codes of 127 throughout: the sum reaches 127 127 2^17."""
    a = lgn.lgn_int8_quantize(torch.ones(130, 1 << 17, device="cuda"))
    b = lgn.lgn_int8_quantize(-torch.ones(140, 1 << 17, device="cuda"))
    check(lgn.lgn_int8_matmul(a, b, out_dtype=torch.float32), product(a, b, torch.float32))


@pytest.mark.parametrize("m,n,k", [(3, 40, 256), (300, 600, 256)])
def test_rows_that_are_not_finite_show(lgn, m, n, k):
    x, w = values(m, k, 1), values(n, k, 2)
    x[1, 5], w[7, 9] = float("inf"), float("nan")
    out = lgn.lgn_int8_matmul(lgn.lgn_int8_quantize(x), lgn.lgn_int8_quantize(w), out_dtype=torch.float32)
    assert out[1].isnan().all() and out[:, 7].isnan().all() and int(out.isnan().sum()) == n + m - 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(5, 24, 64), (400, 300, 128)])
def test_given_outputs(lgn, m, n, k, dtype):
    """Strided and unaligned outputs; what lies around them stays."""
    a, b = lgn.lgn_int8_quantize(values(m, k, 4)), lgn.lgn_int8_quantize(values(n, k, 5))
    for left, right in ((0, 8), (8, 0), (1, 2), (3, 5)):
        whole = torch.full((m + 2, n + left + right), -5.0, dtype=DT[dtype], device="cuda")
        out = whole[1:m + 1, left:left + n]
        assert lgn.lgn_int8_matmul(a, b, out=out) is out
        check(out, product(a, b, DT[dtype]))
        out.fill_(-5.0)
        assert (whole == -5.0).all()


SPANS = [([0, 0, 5, 5, 37, 200, 200], 200), ([3, 10, 10, 300], 310), ([0, 1, 2, 3, 4, 5], 5), ([0, 700, 1501], 1501), ([0, 0, 0], 4), ([2, 40], 60)]


@pytest.mark.parametrize("dtype,bits", [("f32", torch.int32), ("bf16", torch.int64)])
@pytest.mark.parametrize("n,k", [(40, 96), (1000, 640), (129, 2000)])
@pytest.mark.parametrize("ends,rows", SPANS)
def test_grouped_product(lgn, ends, rows, n, k, dtype, bits):
    groups = len(ends) - 1
    a, b = lgn.lgn_int8_quantize(values(rows, k, rows)), lgn.lgn_int8_quantize(values(groups * n, k, n))
    offsets = torch.tensor(ends, dtype=bits, device="cuda")
    want = torch.zeros(rows, n, dtype=torch.float64, device="cuda")
    full = product(a, b, DT[dtype])
    for e in range(groups):
        want[ends[e]:ends[e + 1]] = full[ends[e]:ends[e + 1], e * n:(e + 1) * n]
    check(lgn.lgn_int8_matmul(a, b, out_dtype=DT[dtype], offsets=offsets), want)
    out = torch.full((rows, n), 3.0, dtype=DT[dtype], device="cuda")
    lgn.lgn_int8_matmul(a, b, out=out, offsets=offsets)
    want[:ends[0]] = 3.0
    want[ends[-1]:] = 3.0
    check(out, want)


def test_empty_products(lgn):
    a, b = lgn.lgn_int8_quantize(torch.zeros(5, 0, device="cuda")), lgn.lgn_int8_quantize(torch.zeros(7, 0, device="cuda"))
    assert (lgn.lgn_int8_matmul(a, b) == 0).all()
    a, b = lgn.lgn_int8_quantize(torch.zeros(0, 16, device="cuda")), lgn.lgn_int8_quantize(torch.zeros(7, 16, device="cuda"))
    assert lgn.lgn_int8_matmul(a, b).shape == (0, 7) and lgn.lgn_int8_matmul(b, a).shape == (7, 0)


@pytest.mark.parametrize("rows,k", [(33, 70), (128, 256), (0, 5), (4, 0)])
def test_copied_operands_have_their_own_memory(lgn, rows, k):
    import copy
    import pickle
    a = lgn.lgn_int8_quantize(values(rows, k, 3))
    b = lgn.lgn_int8_quantize(values(24, k, 4))
    want = lgn.lgn_int8_matmul(a, b)
    copies = [copy.deepcopy(a), pickle.loads(pickle.dumps(a))]
    shallow = copy.copy(a)
    assert torch.equal(lgn.lgn_int8_matmul(shallow, b), want)
    a._buffer.fill_(1)
    for c in copies:
        assert (c.rows, c.k) == (rows, k) and torch.equal(lgn.lgn_int8_matmul(c, b), want)
