"""The product's sums, seen past the rounding of a bf16 output: with the negated expected value in the output before an
accumulating call, what is stored is the difference, rounded at 2^-8 of a value that is itself within 2^-8 of nothing.

Bound, with M = sum |a b|: within 1024 k the tensor cores add 32 groups of 32 products, each addition off by at most
2^-23 of the magnitudes so far (truncation included) and the 32 products of a group likewise: (32 + 32) 2^-23 M.  The k / 1024 chunks are
added in fp32 to nearest: (k / 1024) 2^-24 M.  Adding the old value and storing: 2^-24 and 2^-8 of the difference, which is
below 2^-8 M plus the error."""
import pytest
import torch

pytestmark = pytest.mark.gpu

K = 1 << 18


def values(op, k0, k1):
    """What codes k0 .. k1 (multiples of 128) of each row stand for, fp64, on the GPU."""
    pitch = (op.k + 15) // 16 * 16
    v = op.codes[:op.rows * pitch].view(op.rows, pitch)[:, k0:k1].contiguous()
    v = v.view(torch.float8_e4m3fn if op.fmt == 0 else torch.float8_e5m2).double()
    row = torch.arange(op.rows, device="cuda")[:, None]
    blk = torch.arange(k0 // 128, (k1 + 127) // 128, device="cuda")[None]
    at = ((row // 128) * ((op.k + 511) // 512) + blk // 4) * 512 + 16 * (row % 32) + 4 * ((row % 128) // 32) + blk % 4
    return v * torch.exp2(op.scales[at].double() - 127).repeat_interleave(128, 1)[:, :k1 - k0]


def positive(rows, seed, lgn, fmt):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lgn.lgn_fp8_quantize(torch.randn(rows, K, generator=g, device="cuda", dtype=torch.bfloat16).abs_(), fmt)[0]


@pytest.mark.parametrize("odd", [0, 1], ids=["rows of 16 bytes", "odd rows"])
@pytest.mark.parametrize("m,n", [(4, 512), (1024, 1152), (1152, 2048), (2048, 2304)])
def test_sums_over_a_long_contraction(lgn, m, n, odd):
    """Positive operands: what a sum loses at each addition has one sign and shows."""
    a, b = positive(m, 1, lgn, 1), positive(n, 2, lgn, 0)
    want = torch.zeros(m, n, dtype=torch.float64, device="cuda")
    for k in range(0, K, 1 << 14):
        want += values(a, k, k + (1 << 14)) @ values(b, k, k + (1 << 14)).t()
    for dtype in (torch.bfloat16, torch.float32):
        old = (-want).to(torch.bfloat16).to(dtype)
        out = torch.zeros(m, n + 16 + odd, dtype=dtype, device="cuda")[:, :n]
        out.copy_(old)
        lgn.lgn_fp8_matmul(a, b, out=out, accumulate=True)
        tol = (64 * 2.0 ** -23 + (K // 1024) * 2.0 ** -24) * want
        diff = want + old.double()
        half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
        tol = tol + (half + 2.0 ** -24) * (diff.abs() + tol)
        err = (out.double() - diff).abs()
        assert bool((err <= tol).all()), (dtype, float((err / tol).max()), float((err / want).max()))


@pytest.mark.parametrize("positive_only", [False, True])
def test_fp32_sums_at_16384(lgn, positive_only):
    """The figure that the kernel's comment gives for contractions up to 16384: the error's 2-norm below 5e-7 of the output's."""
    k = 16384
    g = torch.Generator(device="cuda").manual_seed(3)
    x, y = (torch.randn(2048, k, generator=g, device="cuda") for _ in range(2))
    if positive_only:
        x, y = x.abs_(), y.abs_()
    a, b = lgn.lgn_fp8_quantize(x, 1)[0], lgn.lgn_fp8_quantize(y, 0)[0]
    want = values(a, 0, k) @ values(b, 0, k).t()
    for m in (2048, 300, 4):                                      # pairs, lone CTAs, shares of k
        sub = lgn.lgn_fp8_quantize(x[:m], 1)[0]
        out = lgn.lgn_fp8_matmul(sub, b, out_dtype=torch.float32)
        assert float((out.double() - want[:m]).norm() / want[:m].norm()) <= 5e-7
