"""The 8-bit quantiser and matrix product against plain fp64 forms.

Quantiser: every code and every scale exactly.  Product: the operands' values are exact in fp64,
so the only errors are those of the fp32 sums and of the last rounding.  The sums run over groups of 32
products; with u = 2^-23 (one unit in the last place, so that truncating additions are covered too) a sum of
G = ceil(k/32) groups of 32 is off by at most (G + 32) u sum |a b|; the last rounding adds half a unit of the
output type."""
import numpy as np
import pytest
import torch

from fp8_helpers import operand_values, quantise, to_np

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def values(rows, cols, seed, dtype, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.exp(spread * torch.randn(rows, cols, generator=g) - 3.0) * torch.where(torch.rand(rows, cols, generator=g) < 0.5, -1.0, 1.0)
    x[torch.rand(rows, cols, generator=g) < 0.2] = 0.0
    return x.to(dtype).cuda()


def check_operand(op, x_np, fmt, square, transpose_of_square=None):
    want, e = quantise(x_np, fmt, square)
    got, ge = operand_values(op)
    if square:
        e = np.repeat(e, 128, axis=0)[:x_np.shape[0]]
    assert np.array_equal(ge, e)
    assert np.array_equal(got, want, equal_nan=True)


SIZES = [(1, 1), (1, 128), (3, 17), (4, 4096), (127, 129), (128, 128), (200, 1000), (300, 513), (513, 300), (64, 2504)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantiser_codes_and_scales(lgn, rows, cols, fmt, dtype):
    x = values(rows, cols, rows * 7 + cols, DT[dtype])
    x_np = to_np(x)
    q, t = lgn.lgn_fp8_quantize(x, fmt)
    assert t is None
    check_operand(q, x_np, fmt, False)
    q, t = lgn.lgn_fp8_quantize(x, fmt, transposed=True)
    check_operand(q, x_np, fmt, False)
    check_operand(t, x_np.T, fmt, False)
    q, t = lgn.lgn_fp8_quantize(x, fmt, rowwise=False, transposed=True)
    assert q is None
    check_operand(t, x_np.T, fmt, False)
    q, t = lgn.lgn_fp8_quantize(x, fmt, lgn.BLOCK_SQUARE, transposed=True)
    check_operand(q, x_np, fmt, True)
    check_operand(t, x_np.T, fmt, True)


@pytest.mark.parametrize("fmt", [0, 1])
def test_quantiser_extremes(lgn, fmt):
    """Block maxima on both sides of every change of exponent, subnormals, the largest floats, ties, all-zero
    blocks, infinities and NaN."""
    top = {0: 448.0, 1: 57344.0}[fmt]
    x = torch.zeros(40, 256)
    for i in range(20):
        x[i, 5] = top * 2.0 ** (i - 10)
        x[i, 6:20] = x[i, 5] * torch.linspace(-1, 1, 14)
        x[i, 133] = float(np.nextafter(np.float32(top * 2.0 ** (i - 10)), np.float32(np.inf)))
    x[20, 0] = torch.finfo(torch.float32).max
    x[21, 0] = 1e-45
    x[22, 0] = 1.1754944e-38
    x[23, :128] = torch.linspace(0, 1e-40, 128)
    x[24, 3] = float("inf"); x[24, 4] = 2.0
    x[25, 3] = float("-inf")
    x[26, 3] = float("nan"); x[26, 200] = -7.0
    x[27, :] = -0.0
    x[28, :128] = 17.0 + torch.arange(128) / 128                            # ties and neighbours once scaled
    x[29, :128] = torch.arange(128) / 16
    for dt in (torch.float32, torch.bfloat16):
        xd = x.to(dt).cuda()
        q, t = lgn.lgn_fp8_quantize(xd, fmt)
        check_operand(q, to_np(xd), fmt, False)
        q, t = lgn.lgn_fp8_quantize(xd, fmt, transposed=True)
        check_operand(q, to_np(xd), fmt, False)
        check_operand(t, to_np(xd).T, fmt, False)
        q, t = lgn.lgn_fp8_quantize(xd, fmt, lgn.BLOCK_SQUARE, transposed=True)
        check_operand(q, to_np(xd), fmt, True)
        check_operand(t, to_np(xd).T, fmt, True)


def test_quantiser_views(lgn):
    """A leading dimension larger than the row, and rows that start at odd addresses."""
    big = values(70, 1000, 3, torch.bfloat16)
    for view in (big[:, :640], big[3:, 1:700], big[::2, 8:136], big[5:6, 3:9]):
        q, t = lgn.lgn_fp8_quantize(view, 0, transposed=True)
        check_operand(q, to_np(view), 0, False)
        check_operand(t, to_np(view).T, 0, False)
        q, _ = lgn.lgn_fp8_quantize(view, 0)
        check_operand(q, to_np(view), 0, False)


def product_bound(av, bv, k, dtype):
    want = av @ bv.T
    mag = np.abs(av) @ np.abs(bv).T
    tol = ((k + 31) // 32 + 32) * 2.0 ** -23 * mag
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    return want, tol + half * (np.abs(want) + tol)


def check_product(out, av, bv, k, add=None):
    want, tol = product_bound(av, bv, k, out.dtype)
    if add is not None:
        half = 2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -24
        want = want + add
        tol = tol + 2 * half * np.abs(want) + 2.0 ** -23 * np.abs(add)
    got = to_np(out)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])


PRODUCTS = [(1, 1, 1), (1, 128, 128), (4, 4096, 512), (5, 333, 1000), (17, 64, 4096), (64, 1000, 2048), (128, 128, 32), (128, 256, 128),
            (130, 200, 300), (257, 513, 640), (777, 2504, 1000), (300, 1, 77), (1000, 40, 1536), (2048, 2048, 256), (1500, 2000, 520)]


@pytest.mark.parametrize("fa,fb,od", [(0, 0, "bf16"), (0, 0, "f32"), (1, 0, "f32"), (0, 1, "bf16"), (1, 1, "f32")])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(lgn, m, n, k, fa, fb, od):
    a, _ = lgn.lgn_fp8_quantize(values(m, k, m + k, torch.float32), fa)
    b, _ = lgn.lgn_fp8_quantize(values(n, k, n + 3 * k, torch.bfloat16), fb, lgn.BLOCK_SQUARE if n % 2 else lgn.BLOCK_ROW)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = lgn.lgn_fp8_matmul(a, b, out_dtype=DT[od], status=status)
    assert int(status.item()) == 0
    check_product(out, operand_values(a)[0], operand_values(b)[0], k)


@pytest.mark.parametrize("fa,fb,od", [(0, 0, "bf16"), (0, 1, "f32")])
@pytest.mark.parametrize("m,n,k", [(3000, 2501, 700), (2049, 4112, 1300), (5000, 1160, 2100), (1111, 5003, 1025)])
def test_large_product(lgn, m, n, k, fa, fb, od):
    """Sizes that take the kernels for large products, in both orientations, with ragged edges; accumulating too."""
    a, _ = lgn.lgn_fp8_quantize(values(m, k, m + k, torch.float32), fa)
    b, _ = lgn.lgn_fp8_quantize(values(n, k, n + 3 * k, torch.bfloat16), fb)
    av, bv = operand_values(a)[0], operand_values(b)[0]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    buf = torch.full((m + 2, n), 7.0, dtype=DT[od], device="cuda")
    out = lgn.lgn_fp8_matmul(a, b, out=buf[1:m + 1], status=status)
    check_product(out, av, bv, k)
    before = to_np(out)
    lgn.lgn_fp8_matmul(a, b, out=out, accumulate=True, status=status)
    check_product(out, av, bv, k, before)
    assert int(status.item()) == 0
    assert bool((buf[0] == 7.0).all()) and bool((buf[-1] == 7.0).all())


@pytest.mark.parametrize("od", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(4, 300, 700), (130, 200, 300), (777, 640, 1000), (1500, 2000, 520), (40, 96, 4096)])
def test_product_accumulates_into_views(lgn, m, n, k, od):
    """accumulate, with an output whose rows are longer than n; what lies between stays untouched."""
    a, _ = lgn.lgn_fp8_quantize(values(m, k, 1, torch.bfloat16), 0)
    b, _ = lgn.lgn_fp8_quantize(values(n, k, 2, torch.bfloat16), 1)
    av, bv = operand_values(a)[0], operand_values(b)[0]
    for lead, off in ((n + 16 - n % 16 + 32, 0), (n + 7, 3)):
        buf = torch.randn(m, lead, device="cuda").to(DT[od])
        before = buf.clone()
        view = buf[:, off:off + n]
        lgn.lgn_fp8_matmul(a, b, out=view, accumulate=True)
        check_product(view, av, bv, k, to_np(before[:, off:off + n]))
        again = before.clone()
        again[:, off:off + n] = buf[:, off:off + n]
        assert torch.equal(again, buf)
        lgn.lgn_fp8_matmul(a, b, out=view)
        check_product(view, av, bv, k)


def test_product_is_the_same_every_time(lgn):
    for m, n, k in ((8, 2048, 4096), (700, 900, 1300)):
        a, _ = lgn.lgn_fp8_quantize(values(m, k, 1, torch.bfloat16), 0)
        b, _ = lgn.lgn_fp8_quantize(values(n, k, 2, torch.bfloat16), 0)
        first = lgn.lgn_fp8_matmul(a, b, out_dtype=torch.float32)
        for _ in range(5):
            assert torch.equal(first, lgn.lgn_fp8_matmul(a, b, out_dtype=torch.float32))


def test_non_finite_entries_reach_their_own_rows_only(lgn):
    x = values(200, 300, 5, torch.float32)
    x[7, 11] = float("inf")
    x[130, 299] = float("nan")
    a, _ = lgn.lgn_fp8_quantize(x, 0)
    b, _ = lgn.lgn_fp8_quantize(values(260, 300, 6, torch.float32), 0)
    for out in (lgn.lgn_fp8_matmul(a, b, out_dtype=torch.float32), lgn.lgn_fp8_matmul(b, a, out_dtype=torch.float32).t()):
        bad = ~torch.isfinite(out)
        want = torch.zeros(200, dtype=torch.bool, device="cuda")
        want[7] = want[130] = True
        assert torch.equal(bad, want[:, None].expand(200, 260))


def test_empty_extents(lgn):
    e = lgn.new_fp8_operand(5, 0, 0, "cuda")
    f = lgn.new_fp8_operand(7, 0, 0, "cuda")
    out = torch.full((5, 7), 3.0, device="cuda")
    lgn.lgn_fp8_matmul(e, f, out=out, accumulate=True)
    assert bool((out == 3.0).all())
    lgn.lgn_fp8_matmul(e, f, out=out)
    assert bool((out == 0.0).all())
    q, _ = lgn.lgn_fp8_quantize(torch.zeros(0, 128, device="cuda"))
    b, _ = lgn.lgn_fp8_quantize(torch.ones(9, 128, device="cuda"))
    assert lgn.lgn_fp8_matmul(q, b).shape == (0, 9)
    assert lgn.lgn_fp8_matmul(b, q).shape == (9, 0)


def test_other_streams(lgn):
    """The quantiser and the product on a stream that is not the current one."""
    x = values(300, 512, 8, torch.bfloat16)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    a, _ = lgn.lgn_fp8_quantize(x, 0, stream=s)
    out = lgn.lgn_fp8_matmul(a, a, out_dtype=torch.float32, stream=s)
    s.synchronize()
    av = operand_values(a)[0]
    check_product(out, av, av, 512)


def test_raw_stream_handles_need_given_outputs(lgn):
    x = torch.ones(4, 256, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with pytest.raises(ValueError):
        lgn.lgn_fp8_quantize(x, stream=s.cuda_stream)
    q = lgn.new_fp8_operand(4, 256, 0, "cuda")
    lgn.lgn_fp8_quantize(x, out=q, stream=s.cuda_stream)
    with pytest.raises(ValueError):
        lgn.lgn_fp8_matmul(q, q, stream=s.cuda_stream)
    out = torch.empty(4, 4, device="cuda")
    lgn.lgn_fp8_matmul(q, q, out=out, stream=s.cuda_stream)
    s.synchronize()
    assert bool((out == 256.0).all())


def test_offsets_beyond_32_bits(lgn):
    """An output of more than 2^32 elements, and an input of which the last rows start beyond 2^32 elements."""
    m, n, k = 66000, 65536, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    a, _ = lgn.lgn_fp8_quantize(torch.randn(m, k, generator=g, device="cuda").bfloat16())
    b, _ = lgn.lgn_fp8_quantize(torch.randn(n, k, generator=g, device="cuda").bfloat16())
    out = lgn.lgn_fp8_matmul(a, b)
    rows = [0, 1, 65535, 65536, 65537, m - 1]
    av, bv = operand_values(a)[0][rows], operand_values(b)[0]
    check_product(out[rows], av, bv, k)
    del out
    x = torch.zeros(2 ** 22 + 8, 1040, dtype=torch.bfloat16, device="cuda")
    x[-5:] = torch.randn(5, 1040, generator=g, device="cuda").bfloat16()
    q, t = lgn.lgn_fp8_quantize(x, 0, transposed=True)
    want, e = quantise(to_np(x[-5:]), 0)
    codes = q.codes[-5 * 1040:].cpu().reshape(5, 1040).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    assert np.array_equal(codes * 2.0 ** np.repeat(e, 128, axis=1)[:, :1040].astype(np.float64), want)
    tail = t.codes.reshape(1040, 2 ** 22 + 16)[:, 2 ** 22 - 120:2 ** 22 + 8].cpu().view(torch.float8_e4m3fn).float().numpy()
    tv, te = quantise(to_np(x[-8:]).T, 0)                       # the block of the last 8 rows
    assert np.array_equal(tail[:, -8:] * 2.0 ** te.astype(np.float64), tv)


def test_refusals(lgn):
    x = torch.ones(4, 256, device="cuda")
    q, _ = lgn.lgn_fp8_quantize(x)
    with pytest.raises(lgn.LgnError):
        lgn.lgn_fp8_quantize(x, 7)
    with pytest.raises(lgn.LgnError):
        lgn.lgn_fp8_quantize(x, 0, 9)
    with pytest.raises(ValueError):
        lgn.lgn_fp8_quantize(x, rowwise=False)
    with pytest.raises(ValueError):
        lgn.lgn_fp8_quantize(x.t())
    with pytest.raises(TypeError):
        lgn.lgn_fp8_quantize(x.half())
    with pytest.raises(ValueError):
        lgn.lgn_fp8_matmul(q, lgn.lgn_fp8_quantize(x[:, :128])[0])
    with pytest.raises(ValueError):
        lgn.lgn_fp8_matmul(q, q, accumulate=True)
    with pytest.raises(ValueError):
        lgn.lgn_fp8_matmul(q, q, out=torch.empty(4, 5, device="cuda"))
    with pytest.raises(ValueError):
        lgn.lgn_fp8_matmul(q._replace(codes=q.codes[:100]), q)
    with pytest.raises(lgn.LgnError):
        lgn.lgn_fp8_matmul(q._replace(fmt=2), q)
    raw = lgn.raw()
    p = x.data_ptr()
    assert raw.lgn_fp8_quantize(p, 4, 256, 255, 0, 0, 0, q.codes.data_ptr(), q.scales.data_ptr(), None, None, None) == 1     # ld < cols
    assert raw.lgn_fp8_quantize(p, 4, 256, 256, 0, 0, 0, q.codes.data_ptr(), None, None, None, None) == 1
    assert raw.lgn_fp8_quantize(p, 4, 256, 256, 0, 0, 0, q.codes.data_ptr() + 8, q.scales.data_ptr(), None, None, None) == 1
    assert raw.lgn_fp8_quantize(p, 4, 256, 256, 0, 0, 0, p, q.scales.data_ptr(), None, None, None) == 1                      # overlap
    assert raw.lgn_fp8_quantize(p, 2 ** 31, 256, 256, 0, 0, 0, q.codes.data_ptr(), q.scales.data_ptr(), None, None, None) == 2
    args = [q.codes.data_ptr(), q.scales.data_ptr(), 0, q.codes.data_ptr(), q.scales.data_ptr(), 0, 4, 4, 256]
    assert raw.lgn_fp8_matmul(*args, p, 3, 0, 0, None, None) == 1                                                             # ldo < n
    assert raw.lgn_fp8_matmul(*args, None, 4, 0, 0, None, None) == 1
    assert raw.lgn_fp8_matmul(*args, p, 4, 5, 0, None, None) == 1
    assert raw.lgn_fp8_matmul(*args, q.codes.data_ptr(), 4, 0, 0, None, None) == 1                                            # out over an operand
