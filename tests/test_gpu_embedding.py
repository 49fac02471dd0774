"""Embedding lookup and table gradient against fp64 forms on the CPU.

Lookup: one product and one rounding, each in fp32 or the output's type: exact up to half a unit of
the product in fp32 and of the output.  Gradient: a sum of m rows in fp32 is off by at most
m 2^-24 sum |dout|, then one product and one rounding (and one addition when it accumulates)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def np64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def make_ids(n, vocab, seed, kind, dtype):
    g = torch.Generator().manual_seed(seed)
    if kind == "uniform":
        ids = torch.randint(0, vocab, (n,), generator=g)
    elif kind == "one":
        ids = torch.full((n,), vocab // 2)
    elif kind == "skewed":
        ids = (torch.rand(n, generator=g) ** 6 * vocab).long().clamp(max=vocab - 1)
    else:                                             # many outside the table, far ones among them
        ids = torch.randint(-vocab, 2 * vocab, (n,), generator=g)
        if n > 3:
            ids[1] = -2 ** 31 if dtype == torch.int32 else -2 ** 62
            ids[2] = 2 ** 31 - 1 if dtype == torch.int32 else 2 ** 40
            ids[3] = vocab
    return ids.to(dtype).cuda()


def check_lookup(out, table, ids, scale):
    t64, i = np64(table), ids.cpu().numpy().astype(np.int64).reshape(-1)
    want = np.zeros((i.size, table.shape[1]))
    inside = (i >= 0) & (i < table.shape[0])
    want[inside] = t64[i[inside]] * float(np.float32(scale))
    got = np64(out)
    assert got.shape == want.shape
    assert np.all(np.abs(got - want) <= (2.0 ** -24 + HALF[out.dtype]) * (1 + 2.0 ** -7) * np.abs(want))
    assert np.all(got[~inside] == 0.0)
    return int((~inside).sum())


@pytest.mark.parametrize("tdt,odt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (1, 100, 4096), (3, 7, 5), (64, 1000, 2048), (513, 50, 270), (1000, 333, 64), (77, 129, 1000), (2000, 64, 8)])
def test_lookup(lgn, n, vocab, dim, tdt, odt):
    table = torch.randn(vocab, dim, generator=torch.Generator().manual_seed(1)).to(DT[tdt]).cuda()
    for kind, idt in (("uniform", torch.int64), ("outside", torch.int64), ("outside", torch.int32)):
        ids = make_ids(n, vocab, n, kind, idt)
        count = torch.full((1,), 5, dtype=torch.int64, device="cuda")
        out = lgn.lgn_embedding(table, ids, 45.25, out_dtype=DT[odt], n_outside=count)
        assert out.dtype == DT[odt]
        assert check_lookup(out, table, ids, 45.25) == int(count.item()) - 5
        assert torch.equal(out, lgn.lgn_embedding(table, ids, 45.25, out_dtype=DT[odt]))


@pytest.mark.parametrize("odt", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [8, 9, 10, 11, 15, 17, 33, 100, 257, 999])
def test_lookup_without_gaps_at_any_address(lgn, dim, odt):
    """Outputs of odd rows without gaps, at every element offset from a 16-byte boundary, and what lies around them."""
    table = torch.randn(60, dim, device="cuda")
    for n in (1, 2, 130, 1111):
        ids = make_ids(n, 60, n + dim, "outside", torch.int64)
        for off in range(9):
            buf = torch.full((n * dim + 40,), 7.0, dtype=DT[odt], device="cuda")
            view = buf[off:off + n * dim].view(n, dim)
            count = torch.zeros(1, dtype=torch.int64, device="cuda")
            lgn.lgn_embedding(table, ids, -3.0, out=view, n_outside=count)
            assert check_lookup(view, table, ids, -3.0) == int(count.item())
            assert bool((buf[:off] == 7.0).all()) and bool((buf[off + n * dim:] == 7.0).all())


def test_lookup_keeps_bits_at_scale_one(lgn):
    table = torch.randn(40, 128, device="cuda")
    table[3, 7], table[3, 8], table[3, 9] = float("inf"), float("nan"), -0.0
    ids = torch.tensor([3, 39, 0, 3], device="cuda")
    out = lgn.lgn_embedding(table, ids)
    assert torch.equal(out.view(torch.int32), table[ids].view(torch.int32))


def test_lookup_views(lgn):
    """Rows further apart than their length, rows that start at odd addresses, an output inside a larger one."""
    big = torch.randn(200, 700, device="cuda")
    for tdt in DT.values():
        for table in (big.to(tdt)[:, :640], big.to(tdt)[:, 1:514], big.to(tdt)[::3, 4:260]):
            ids = make_ids(90, table.shape[0], 4, "outside", torch.int64).reshape(9, 10)
            buf = torch.full((90, 1000), 7.0, device="cuda")
            for off in (0, 3, 8):
                buf.fill_(7.0)
                view = buf[:, off:off + table.shape[1]]
                lgn.lgn_embedding(table, ids, 2.0, out=view)
                check_lookup(view, table, ids, 2.0)
                assert bool((buf[:, :off] == 7.0).all()) and bool((buf[:, off + table.shape[1]:] == 7.0).all())


def check_grad(got, dout, ids, vocab, scale, padding, before=None):
    d, i = np64(dout), ids.cpu().numpy().astype(np.int64).reshape(-1)
    keep = (i >= 0) & (i < vocab) & (i != padding)
    want, mag, cnt = (np.zeros((vocab, d.shape[1])) for _ in range(3))
    np.add.at(want, i[keep], d[keep])
    np.add.at(mag, i[keep], np.abs(d[keep]))
    np.add.at(cnt, i[keep], 1.0)
    s = float(np.float32(scale))
    want, mag = want * s, mag * abs(s)
    tol = (cnt + 1) * 2.0 ** -24 * mag * (1 + 1e-5)
    if before is not None:
        want = want + before
        tol = tol + 2.0 ** -24 * (np.abs(want) + tol)
    tol = tol + HALF[got.dtype] * (np.abs(want) + tol)
    g = np64(got)
    bad = ~(np.abs(g - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], g[bad][:4], want[bad][:4])
    absent = cnt[:, 0] == 0
    assert np.array_equal(g[absent], (np.zeros_like(g) if before is None else before)[absent])


@pytest.mark.parametrize("ddt,odt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("kind", ["uniform", "one", "skewed", "outside"])
@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (1, 500, 64), (31, 7, 5), (33, 40, 256), (700, 1000, 270), (4999, 3001, 40), (20000, 515, 24), (9001, 70001, 8)])
def test_gradient(lgn, n, vocab, dim, kind, ddt, odt):
    g = torch.Generator().manual_seed(n)
    dout = torch.randn(n, dim, generator=g).to(DT[ddt]).cuda()
    ids = make_ids(n, vocab, n + 1, kind, torch.int32 if n % 2 else torch.int64)
    pad = int(ids[0].item()) if kind == "skewed" else -1
    got = lgn.lgn_embedding_grad(dout, ids, vocab, 0.75, padding_idx=pad, out_dtype=DT[odt])
    check_grad(got, dout, ids, vocab, 0.75, pad)
    ws = torch.full((lgn.new_embedding_grad_workspace(n, vocab, dim, "cuda").numel(),), 0xEE, dtype=torch.uint8, device="cuda")
    assert torch.equal(got, lgn.lgn_embedding_grad(dout, ids, vocab, 0.75, padding_idx=pad, out_dtype=DT[odt], ws=ws))
    out = torch.randn(vocab, dim, device="cuda").to(DT[odt])
    before = np64(out)
    lgn.lgn_embedding_grad(dout, ids, vocab, 0.75, padding_idx=pad, out=out, accumulate=True, ws=ws)
    check_grad(out, dout, ids, vocab, 0.75, pad, before)


@pytest.mark.parametrize("n", [2, 1023, 1024, 1025, 1500, 2048, 2049, 3000, 4095, 4096, 4097, 8193])
def test_gradient_at_the_sorts_edges(lgn, n):
    """Both sorts, at the sizes where one form ends and the next begins; ids that come many times and once."""
    dout = torch.randn(n, 6, generator=torch.Generator().manual_seed(n)).cuda()
    for vocab, kind in ((13, "uniform"), (70001, "skewed")):
        for idt in (torch.int32, torch.int64):
            ids = make_ids(n, vocab, n, kind, idt)
            got = lgn.lgn_embedding_grad(dout, ids, vocab, padding_idx=3)
            check_grad(got, dout, ids, vocab, 1.0, 3)
            assert torch.equal(got, lgn.lgn_embedding_grad(dout, ids, vocab, padding_idx=3))


def test_gradient_wide_keys(lgn):
    """More than 18 bits of ids: three passes of the sort."""
    vocab, n = 600_011, 3000
    dout = torch.randn(n, 3, device="cuda")
    ids = make_ids(n, vocab, 9, "uniform", torch.int64)
    ids[::7] = vocab - 1
    check_grad(lgn.lgn_embedding_grad(dout, ids, vocab), dout, ids, vocab, 1.0, -1)


def test_gradient_views_and_nothing(lgn):
    big = torch.randn(300, 520, device="cuda")
    ids = make_ids(100, 50, 3, "uniform", torch.int64)
    for off, lead in ((0, 520), (8, 528), (1, 521)):
        dout = big[::3, off:off + 512]
        buf = torch.full((50, lead), 7.0, device="cuda")
        view = buf[:, lead - 512:]
        lgn.lgn_embedding_grad(dout, ids, 50, out=view)
        check_grad(view, dout, ids, 50, 1.0, -1)
        assert bool((buf[:, :lead - 512] == 7.0).all())
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    got = lgn.lgn_embedding_grad(torch.zeros(0, 16, device="cuda"), none, 9)
    assert got.shape == (9, 16) and bool((got == 0).all())
    assert lgn.lgn_embedding_grad(torch.zeros(4, 0, device="cuda"), none.new_zeros(4), 9).shape == (9, 0)
    assert lgn.lgn_embedding(torch.zeros(9, 16, device="cuda"), none).shape == (0, 16)
    out = lgn.lgn_embedding(torch.zeros(0, 16, device="cuda"), none.new_zeros(5))
    assert out.shape == (5, 16) and bool((out == 0).all())


def test_gradient_is_that_of_the_lookup(lgn):
    """<lookup(E + h D) - lookup(E - h D), G> / 2h = <gradient(G), D>: the lookup is linear in the table, so the
    difference is exact up to the rounding of the two lookups (half a unit of fp32 of values of order 10)."""
    g = torch.Generator(device="cuda").manual_seed(2)
    vocab, dim, n = 97, 72, 400
    e = torch.randn(vocab, dim, generator=g, device="cuda", dtype=torch.float64)
    d = torch.randn(vocab, dim, generator=g, device="cuda", dtype=torch.float64)
    up = torch.randn(n, dim, generator=g, device="cuda")
    ids = make_ids(n, vocab, 5, "outside", torch.int64)
    h = 0.5
    hi, lo = (lgn.lgn_embedding((e + s * h * d).float(), ids, 3.0).double() for s in (1, -1))
    left = float(((hi - lo) * up.double()).sum()) / (2 * h)
    grad = lgn.lgn_embedding_grad(up, ids, vocab, 3.0).double()
    right = float((grad * d).sum())
    mag = float((up.double().abs() * 3.0 * 8.0).sum())
    assert abs(left - right) <= 4 * 2.0 ** -24 * mag


def test_other_streams(lgn):
    table = torch.randn(100, 64, device="cuda")
    ids = make_ids(50, 100, 3, "uniform", torch.int64)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = lgn.lgn_embedding(table, ids, stream=s)
    s.synchronize()
    check_lookup(out, table, ids, 1.0)
    ws = lgn.new_embedding_grad_workspace(50, 100, 64, "cuda")
    got = lgn.lgn_embedding_grad(out, ids, 100, ws=ws, stream=s)
    s.synchronize()
    check_grad(got, out, ids, 100, 1.0, -1)


def test_offsets_beyond_32_bits(lgn):
    """A table and its gradient of more than 2^32 elements."""
    vocab, dim = 2 ** 21 + 3, 2056
    table = torch.zeros(vocab, dim, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, vocab - 1, 2 ** 21, 5, vocab - 1, 2 ** 20], device="cuda")
    table[rows] = torch.randn(6, dim, device="cuda").bfloat16()
    ids = torch.cat([rows, torch.tensor([vocab, -1], device="cuda")])
    out = lgn.lgn_embedding(table, ids)
    assert torch.equal(out[:6], table[rows]) and bool((out[6:] == 0).all())
    dout = torch.randn(8, dim, device="cuda")
    table.fill_(7.0)
    lgn.lgn_embedding_grad(dout, ids, vocab, out=table)
    check_grad(table[rows.unique()], dout[:6], torch.unique(rows, return_inverse=True)[1], rows.unique().numel(), 1.0, -1)
    assert int((table != 0).any(dim=1).sum()) == rows.unique().numel()


def test_raw_stream_handles_need_given_memory(lgn):
    table = torch.randn(10, 16, device="cuda")
    ids = torch.tensor([3, 4], device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with pytest.raises(ValueError):
        lgn.lgn_embedding(table, ids, stream=s.cuda_stream)
    out = torch.empty(2, 16, device="cuda")
    lgn.lgn_embedding(table, ids, out=out, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(out, table[ids])
    with pytest.raises(ValueError):
        lgn.lgn_embedding_grad(out, ids, 10, out=torch.empty(10, 16, device="cuda"), stream=s.cuda_stream)


def test_refusals(lgn):
    table = torch.zeros(10, 16, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    with pytest.raises(TypeError):
        lgn.lgn_embedding(table, ids.float())
    with pytest.raises(TypeError):
        lgn.lgn_embedding(table.half(), ids)
    with pytest.raises(ValueError):
        lgn.lgn_embedding(table.t(), ids)
    with pytest.raises(ValueError):
        lgn.lgn_embedding(table, ids, out=torch.zeros(4, 15, device="cuda"))
    with pytest.raises(ValueError):
        lgn.lgn_embedding(table, ids[::2])
    with pytest.raises(lgn.LgnError):
        lgn.lgn_embedding(table, ids, out=table[:4])                             # overlap
    with pytest.raises(ValueError):
        lgn.lgn_embedding_grad(table, ids, 10)
    with pytest.raises(ValueError):
        lgn.lgn_embedding_grad(table[:4], ids, 10, accumulate=True)
    with pytest.raises(lgn.LgnError) as e:
        lgn.lgn_embedding_grad(table[:4], ids, 10, ws=torch.zeros(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 3
    raw = lgn.raw()
    o = torch.zeros(4, 16, device="cuda")
    assert raw.lgn_embedding(table.data_ptr(), 10, 16, 15, 0, ids.data_ptr(), 64, 4, 1.0, o.data_ptr(), 16, 0, None, None) == 1
    assert raw.lgn_embedding(table.data_ptr(), 10, 16, 16, 0, ids.data_ptr(), 16, 4, 1.0, o.data_ptr(), 16, 0, None, None) == 1
    assert raw.lgn_embedding(table.data_ptr(), 2 ** 31, 16, 16, 0, ids.data_ptr(), 64, 4, 1.0, o.data_ptr(), 16, 0, None, None) == 2
    assert raw.lgn_embedding(table.data_ptr() + 2, 10, 16, 16, 0, ids.data_ptr(), 64, 4, 1.0, o.data_ptr(), 16, 0, None, None) == 1
