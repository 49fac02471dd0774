"""The grouped products, 8-bit integers and the distillation loss where offsets pass 32 bits: what stands at the far end equals what
a small call gives."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def release():
    yield
    torch.cuda.empty_cache()


def tail(rows, cols, keep, seed, dtype=torch.bfloat16):
    """A matrix of zeros but for its last `keep` rows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.zeros(rows, cols, dtype=dtype, device="cuda")
    t[-keep:] = torch.randn(keep, cols, generator=g, device="cuda").to(dtype)
    return t


def test_int8_rows(lgn):
    x = tail(70000, 32768, 3, 1)                                               # 2.3e9 values and codes
    q = lgn.lgn_int8_quantize(x)
    small = lgn.lgn_int8_quantize(x[-3:].contiguous())
    assert torch.equal(q.codes[-3:], small.codes) and torch.equal(q.scales[-3:], small.scales)
    w = lgn.lgn_int8_quantize(tail(40, 32768, 40, 2))
    assert torch.equal(lgn.lgn_int8_matmul(q, w, out_dtype=torch.float32)[-3:], lgn.lgn_int8_matmul(small, w, out_dtype=torch.float32))


def test_int8_output(lgn):
    a, b = (lgn.lgn_int8_quantize(tail(n, 64, 200, i)) for i, n in enumerate((70000, 33000)))       # 2.3e9 results
    y = lgn.lgn_int8_matmul(a, b)
    want = (a.codes[-200:].double() @ b.codes[-200:].double().t() * a.scales[-200:, None].double() * b.scales[-200:].double())
    assert bool(((y[-200:, -200:].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -20)).all())
    assert not y[:300].any()


@pytest.mark.parametrize("transposed", [False, True])
def test_grouped_rows_and_weights(lgn, transposed):
    rows, k, n, groups = 300000, 8192, 8192, 40                                 # 2.5e9 inputs and outputs, 2.7e9 weights
    x = tail(rows, k, 100, 1)
    w = torch.zeros(groups, n, k, dtype=torch.bfloat16, device="cuda")
    w[-1] = tail(n, k, n, 2)
    offsets = torch.tensor([0] + [rows - 500] * (groups - 1) + [rows], device="cuda")
    y = lgn.lgn_grouped_matmul(x, w, offsets, transposed=transposed)
    want = x[-100:].double() @ (w[-1].double() if transposed else w[-1].double().t())
    mag = x[-100:].double().abs() @ (w[-1].double().abs() if transposed else w[-1].double().abs().t())
    tol = 1.1e-6 * mag + 2.0 ** -19 * mag                                      # the tensor cores' additions; sums of 16 chunks and their rounding
    assert bool(((y[-100:].double() - want).abs() <= tol + 2.0 ** -8 * (want.abs() + tol)).all())
    assert not y[:1000].any() and not y[-500:-100].any()


def test_grouped_gradient(lgn):
    groups, m, n = 40, 8192, 8192                                              # 2.7e9 outputs
    dy, x = tail(300, m, 300, 1), tail(300, n, 300, 2)
    offsets = torch.tensor([0, 100] + [100] * (groups - 2) + [300], device="cuda")
    out = lgn.lgn_grouped_weight_grad(dy, x, offsets, out_dtype=torch.bfloat16)
    for e, a, b in ((0, 0, 100), (groups - 1, 100, 300)):
        small = lgn.lgn_grouped_weight_grad(dy[a:b].contiguous(), x[a:b].contiguous(), torch.tensor([0, b - a], device="cuda"), out_dtype=torch.bfloat16)
        want, mag = dy[a:b].double().t() @ x[a:b].double(), dy[a:b].double().abs().t() @ x[a:b].double().abs()
        for got in (out[e], small[0]):
            tol = 1.1e-6 * mag
            assert bool(((got.double() - want).abs() <= tol + 2.0 ** -8 * (want.abs() + tol)).all())
    assert not out[1:-1].any()


def test_aligned_copies(lgn):
    x = tail(60001, 40001, 2, 1)                                               # 2.4e9 values at odd rows
    w = tail(8, 40001, 8, 2)[None]
    offsets = torch.tensor([0, 60001], device="cuda")
    got = lgn.lgn_grouped_matmul(x, w, offsets, out_dtype=torch.float32)[-2:]
    want, mag = x[-2:].double() @ w[0].double().t(), x[-2:].double().abs() @ w[0].double().abs().t()
    assert bool(((got.double() - want).abs() <= (1.1e-6 + 80 * 2.0 ** -24) * mag).all())       # 79 chunks added in fp32


@pytest.mark.parametrize("in_place", [False, True])
def test_distill_rows(lgn, in_place):
    t, v = 20000, 131072                                                        # 2.6e9 logits
    s = tail(t, v, 4, 1)
    ids = torch.randint(0, v, (t, 8), device="cuda")
    z, labels = torch.randn(t, 8, device="cuda"), torch.randint(0, v, (t,), device="cuda")
    last = s[-4:].clone()
    want, d = lgn.lgn_distill_loss(last, ids[-4:], z[-4:], labels[-4:].clone(), 2.0, 0.5, grad=True)
    loss, got = lgn.lgn_distill_loss(s, ids, z, labels, 2.0, 0.5, grad=True, dlogits=s if in_place else None)
    tol = 2.0 ** -7 * d.double().abs() + 1e-9                                  # two roundings to bf16, and 400 2^-24 in fp32 of values of 1e-5; a row may be shared out differently
    assert bool(((got[-4:].double() - d.double()).abs() <= tol).all()) and bool(((loss[-4:] - want).abs() <= 1e-4 * want.abs()).all())
