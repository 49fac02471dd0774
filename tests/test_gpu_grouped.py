"""Products of rows grouped by expert in bf16 against fp64.

The operands are exact in fp64, so the only errors are those of the fp32 sums and of the last rounding.  The tensor cores add groups of 16
products; with u = 2^-23 (one unit in the last place, so that truncating additions are covered too) a sum of G = ceil(k / 16) groups is off
by at most (G + 32) u sum |a b|; the last rounding adds half a unit of the output type."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def values(*shape, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.exp(1.5 * torch.randn(*shape, generator=g) - 3.0) * torch.where(torch.rand(*shape, generator=g) < 0.5, -1.0, 1.0)
    x[torch.rand(*shape, generator=g) < 0.2] = 0.0
    return x.to(torch.bfloat16).cuda()


def check(out, want, mag, k, extra=0.0):
    tol = ((k + 15) // 16 + 32) * 2.0 ** -23 * mag + extra
    tol = tol + HALF[out.dtype] * (want.abs() + tol)
    bad = ~((out.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4], out[bad][:4], want[bad][:4])


def forward(x, w, ends, transposed):
    """(product, sum of magnitudes); zeros in rows of no group."""
    n = w.shape[2 if transposed else 1]
    want, mag = (torch.zeros(x.shape[0], n, dtype=torch.float64, device="cuda") for _ in range(2))
    for e in range(len(ends) - 1):
        we = w[e].double() if transposed else w[e].double().t()
        xe = x[ends[e]:ends[e + 1]].double()
        want[ends[e]:ends[e + 1]] = xe @ we
        mag[ends[e]:ends[e + 1]] = xe.abs() @ we.abs()
    return want, mag


def spans(rows, groups, seed):
    """Ragged ends with empty groups."""
    g = torch.Generator().manual_seed(seed)
    cut = torch.sort(torch.randint(0, rows + 1, (groups - 1,), generator=g)).values.tolist()
    if groups > 3:
        cut[1] = cut[0]
    return [0] + cut + [rows]


SMALL = [([0, 0, 5, 5, 37, 200, 200], 200), ([3, 10, 10, 300], 310), ([0, 1, 2, 3, 4, 5], 5), ([0, 700, 1501], 1501), ([0, 0, 0], 4), ([2, 40], 60), ([0, 1], 1)]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype,bits", [("f32", torch.int32), ("bf16", torch.int64)])
@pytest.mark.parametrize("n,k", [(1, 8), (40, 96), (1000, 640), (129, 2001), (264, 1096)])
@pytest.mark.parametrize("ends,rows", SMALL)
def test_product(lgn, ends, rows, n, k, dtype, bits, transposed):
    groups = len(ends) - 1
    x, w = values(rows, k, seed=rows), values(groups, *((k, n) if transposed else (n, k)), seed=n)
    offsets = torch.tensor(ends, dtype=bits, device="cuda")
    want, mag = forward(x, w, ends, transposed)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    check(lgn.lgn_grouped_matmul(x, w, offsets, out_dtype=DT[dtype], transposed=transposed, status=status), want, mag, k)
    out = torch.full((rows, n), 3.0, dtype=DT[dtype], device="cuda")
    assert lgn.lgn_grouped_matmul(x, w, offsets, out=out, transposed=transposed, status=status) is out
    check(out[ends[0]:ends[-1]], want[ends[0]:ends[-1]], mag[ends[0]:ends[-1]], k)
    assert (out[:ends[0]] == 3.0).all() and (out[ends[-1]:] == 3.0).all() and int(status.item()) == 0


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows,groups,n,k,dtype", [(3000, 3, 2504, 1400, "bf16"), (4001, 40, 512, 264, "f32"), (9000, 5, 1024, 2048, "f32"), (700, 150, 136, 1200, "bf16"),
                                                   (64, 33, 2048, 512, "bf16"), (5000, 2, 777, 1023, "bf16")])
def test_large_product(lgn, rows, groups, n, k, dtype, transposed):
    x, w = values(rows, k, seed=rows), values(groups, *((k, n) if transposed else (n, k)), seed=n)
    ends = spans(rows, groups, k)
    want, mag = forward(x, w, ends, transposed)
    out = lgn.lgn_grouped_matmul(x, w, torch.tensor(ends, device="cuda"), out_dtype=DT[dtype], transposed=transposed)
    check(out, want, mag, k)


def gradient(dy, x, ends):
    want, mag = [], []
    for e in range(len(ends) - 1):
        d, y = dy[ends[e]:ends[e + 1]].double(), x[ends[e]:ends[e + 1]].double()
        want.append(d.t() @ y)
        mag.append(d.abs().t() @ y.abs())
    return torch.stack(want), torch.stack(mag)


@pytest.mark.parametrize("dtype,bits", [("f32", torch.int32), ("bf16", torch.int64)])
@pytest.mark.parametrize("m,n", [(1, 8), (40, 96), (264, 640), (129, 201), (1000, 300)])
@pytest.mark.parametrize("ends,rows", SMALL)
def test_weight_gradient(lgn, ends, rows, m, n, dtype, bits):
    dy, x = values(rows, m, seed=rows), values(rows, n, seed=n)
    for t in (dy, x):                                  # rows of no group must not matter
        t[:ends[0]] = float("nan")
        t[ends[-1]:] = float("inf")
    offsets = torch.tensor(ends, dtype=bits, device="cuda")
    want, mag = gradient(dy, x, ends)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = lgn.lgn_grouped_weight_grad(dy, x, offsets, out_dtype=DT[dtype], status=status)
    check(out, want, mag, rows)
    before = values(len(ends) - 1, m, n, seed=9).to(DT[dtype])
    out = before.clone()
    assert lgn.lgn_grouped_weight_grad(dy, x, offsets, out=out, accumulate=True, status=status) is out
    check(out, want + before.double(), mag + before.double().abs(), rows)
    assert int(status.item()) == 0


@pytest.mark.parametrize("rows,groups,m,n,dtype", [(3000, 3, 2504, 1400, "bf16"), (4001, 40, 512, 264, "f32"), (9000, 5, 1024, 2048, "f32"), (700, 150, 136, 1200, "bf16"),
                                                   (64, 33, 2048, 512, "bf16"), (5000, 2, 777, 1023, "f32")])
def test_large_weight_gradient(lgn, rows, groups, m, n, dtype):
    dy, x = values(rows, m, seed=rows), values(rows, n, seed=n)
    ends = spans(rows, groups, m)
    want, mag = gradient(dy, x, ends)
    check(lgn.lgn_grouped_weight_grad(dy, x, torch.tensor(ends, device="cuda"), out_dtype=DT[dtype]), want, mag, rows)


@pytest.mark.parametrize("rows,m,n", [(900, 264, 520), (6000, 1032, 2048)])
def test_neighbouring_groups_do_not_mix(lgn, rows, m, n):
    """Every other group is NaN: the groups between come out right, whatever their length."""
    lengths = [1, 15, 16, 17, 63, 64, 65, 3, 128, 0, 31, 100]
    ends = [0]
    for i in range(60):
        ends.append(min(rows, ends[-1] + lengths[i % len(lengths)]))
    dy, x, w = values(rows, m, seed=1), values(rows, n, seed=2), values(60, m, n, seed=3)
    for e in range(0, 60, 2):
        dy[ends[e]:ends[e + 1]], x[ends[e]:ends[e + 1]] = float("nan"), float("inf")
    offsets = torch.tensor(ends, device="cuda")
    want, mag = gradient(dy, x, ends)
    got = lgn.lgn_grouped_weight_grad(dy, x, offsets)
    odd = torch.arange(1, 60, 2, device="cuda")
    check(got[odd], want[odd], mag[odd], rows)
    want, mag = forward(dy, w, ends, True)
    got = lgn.lgn_grouped_matmul(dy, w, offsets, transposed=True, out_dtype=torch.float32)
    for e in range(1, 60, 2):
        s = slice(ends[e], ends[e + 1])
        check(got[s], want[s], mag[s], m)


def test_offsets_outside_the_rows(lgn):
    """Counted as the nearest row; one below an earlier one as that one: nothing is read or written outside."""
    x, w = values(100, 64, seed=1), values(4, 72, 64, seed=2)
    for given, ends in (([-5, 20, 10, 90, 500], [0, 20, 20, 90, 100]), ([40, 30, 20, 10, 0], [40] * 5), ([2 ** 40, 0, 0, 0, 7], [100] * 5), ([-2 ** 40, 0, 50, 50, 2 ** 40], [0, 0, 50, 50, 100])):
        offsets = torch.tensor(given, device="cuda")
        want, mag = forward(x, w, ends, False)
        check(lgn.lgn_grouped_matmul(x, w, offsets, out_dtype=torch.float32), want, mag, 64)
        want, mag = gradient(x, x, ends)
        check(lgn.lgn_grouped_weight_grad(x, x, offsets), want, mag, 100)


def test_strides(lgn):
    """Operands and outputs inside larger tensors, at odd addresses, transposed, broadcast; what lies around outputs stays."""
    ends = [0, 30, 30, 170, 300]
    offsets = torch.tensor(ends, device="cuda")
    big, stack = values(310, 700, seed=1), values(4, 300, 700, seed=2)
    shared = values(1, 200, 128, seed=3).expand(4, 200, 128)
    for x, w in ((big[5:305, 8:520], stack[:, 40:240, 16:528]), (big[:300, 3:260], stack[:, ::2, 1:258]), (big[:300, :200], stack.transpose(1, 2)[:, :300, 10:210]), (big[:300, :128], shared)):
        want, mag = forward(x, w, ends, False)
        check(lgn.lgn_grouped_matmul(x, w, offsets), want, mag, x.shape[1])
        wt = w.transpose(1, 2)
        check(lgn.lgn_grouped_matmul(x, wt, offsets, transposed=True), want, mag, x.shape[1])
        for dtype, left, right in ((torch.float32, 4, 8), (torch.bfloat16, 1, 2), (torch.float32, 3, 2)):
            n = w.shape[1]
            whole = torch.full((302, n + left + right), -5.0, dtype=dtype, device="cuda")
            lgn.lgn_grouped_matmul(x, w, offsets, out=whole[1:301, left:left + n])
            check(whole[1:301, left:left + n], want, mag, x.shape[1])
            whole[1:301, left:left + n] = -5.0
            assert (whole == -5.0).all()
    want, mag = gradient(big[:300, :130], big[:300, 200:333], ends)
    for dtype, top, left, right in ((torch.float32, 0, 4, 7), (torch.bfloat16, 2, 1, 2), (torch.float32, 1, 3, 3)):
        whole = torch.full((5, 130 + top, 133 + left + right), -5.0, dtype=dtype, device="cuda")
        out = whole[:4, top:, left:left + 133]
        lgn.lgn_grouped_weight_grad(big[:300, :130], big[:300, 200:333], offsets, out=out)
        check(out, want, mag, 300)
        out.fill_(-5.0)
        assert (whole == -5.0).all()


def test_empty(lgn):
    off = torch.tensor([0, 0, 3], device="cuda")
    bf = dict(dtype=torch.bfloat16, device="cuda")
    assert (lgn.lgn_grouped_matmul(torch.zeros(3, 0, **bf), torch.zeros(2, 5, 0, **bf), off) == 0).all()
    assert lgn.lgn_grouped_matmul(torch.zeros(0, 16, **bf), torch.zeros(2, 5, 16, **bf), off).shape == (0, 5)
    assert lgn.lgn_grouped_matmul(torch.zeros(3, 16, **bf), torch.zeros(2, 0, 16, **bf), off).shape == (3, 0)
    got = lgn.lgn_grouped_weight_grad(torch.zeros(0, 16, **bf), torch.zeros(0, 8, **bf), off)
    assert got.shape == (2, 16, 8) and (got == 0).all()
    assert lgn.lgn_grouped_weight_grad(torch.zeros(3, 0, **bf), torch.zeros(3, 8, **bf), off).shape == (2, 0, 8)


def test_streams_and_graphs(lgn):
    """On another stream, and captured with offsets that change between replays."""
    x, w, dy = values(500, 256, seed=1), values(6, 384, 256, seed=2), values(500, 384, seed=3)
    offsets = torch.tensor(spans(500, 6, 1), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = lgn.lgn_grouped_matmul(x, w, offsets, stream=side)
    side.synchronize()
    check(y, *forward(x, w, offsets.tolist(), False), 256)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dw = lgn.lgn_grouped_matmul(x, w, offsets), lgn.lgn_grouped_weight_grad(dy, x, offsets)
    for seed in range(4):
        offsets.copy_(torch.tensor(spans(500, 6, seed)))
        graph.replay()
        check(y, *forward(x, w, offsets.tolist(), False), 256)
        check(dw, *gradient(dy, x, offsets.tolist()), 500)


def test_same_bits_every_time(lgn):
    x, w = values(333, 4096, seed=1), values(7, 512, 4096, seed=2)
    offsets = torch.tensor(spans(333, 7, 3), device="cuda")
    first = lgn.lgn_grouped_matmul(x, w, offsets, out_dtype=torch.float32)
    for _ in range(5):
        assert torch.equal(lgn.lgn_grouped_matmul(x, w, offsets, out_dtype=torch.float32), first)


@pytest.mark.parametrize("rows,groups,m,n,dtype", [(5000, 1, 100, 72, "f32"), (20000, 2, 200, 301, "f32"), (4001, 4, 256, 512, "bf16"), (9000, 8, 128, 128, "f32"), (700, 3, 129, 40, "bf16")])
def test_weight_gradient_of_few_tiles(lgn, rows, groups, m, n, dtype):
    """Small matrices, long groups of uneven and empty sizes: rows are shared out among CTAs."""
    dy, x = values(rows, m, seed=rows), values(rows, n, seed=n)
    ends = spans(rows, groups, m)
    want, mag = gradient(dy, x, ends)
    offsets = torch.tensor(ends, device="cuda")
    check(lgn.lgn_grouped_weight_grad(dy, x, offsets, out_dtype=DT[dtype]), want, mag, rows)
    before = values(groups, m, n, seed=9).to(DT[dtype])
    out = before.clone()
    lgn.lgn_grouped_weight_grad(dy, x, offsets, out=out, accumulate=True)
    check(out, want + before.double(), mag + before.double().abs(), rows)


def test_align_rows(lgn):
    """Values and the zeros behind them, for rows at any boundary; what lies behind the copy stays."""
    big = values(7, 40, 333, seed=4)
    for view in (big[:, :, :3], big[1:4, 5:30, 7:300], big[:1, :1, 1:332], big[:, ::3, 1:9], big[::2, :, :332]):
        g, r, c = view.shape
        pitch = (c + 7) // 8 * 8
        out = torch.full((g * r * pitch + 16,), -7.0, dtype=torch.bfloat16, device="cuda")
        assert lgn.raw().lgn_align_rows(view.data_ptr(), view.stride(1), view.stride(0), g, r, c, out.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
        got = out[:-16].view(g, r, pitch)
        assert torch.equal(got[..., :c], view) and not got[..., c:].any() and (out[-16:] == -7.0).all()
