"""Plain fp64 forms of the 8-bit quantiser and of what its codes stand for, on the CPU, for the
tests: written from the formats' definitions, value by value."""
import numpy as np
import torch

FMAX = {0: 448.0, 1: 57344.0}          # E4M3, E5M2
MAN = {0: 3, 1: 2}
EMIN = {0: -6, 1: -14}


def to_np(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def block_exponent(amax, fmt):
    """Smallest integer e >= -127 with amax 2^-e <= fmax, by trial."""
    if amax == 0.0:
        return -127
    e = int(np.floor(np.log2(amax))) - 20
    while amax * 2.0 ** -e > FMAX[fmt]:
        e += 1
    return max(e, -127)


def round8(y, fmt):
    """Nearest value of the format, ties to even; NaN for non-finite."""
    out = np.full_like(y, np.nan)
    f = np.isfinite(y)
    a = np.abs(y[f])
    ex = np.floor(np.log2(np.maximum(a, 2.0 ** EMIN[fmt])))
    step = 2.0 ** (np.maximum(ex, EMIN[fmt]) - MAN[fmt])
    out[f] = np.sign(y[f]) * np.rint(a / step) * step
    return out


def quantise(x, fmt, square=False):
    """(values the codes stand for, exponents [rows or row blocks, column blocks]) of a 2-d array."""
    r, c = x.shape
    rb = 128 if square else 1
    vals = np.zeros_like(x)
    exps = np.zeros(((r + rb - 1) // rb, (c + 127) // 128), dtype=np.int64)
    for i in range(exps.shape[0]):
        for j in range(exps.shape[1]):
            b = x[i * rb:(i + 1) * rb, j * 128:(j + 1) * 128]
            fin = np.abs(b[np.isfinite(b)])
            e = block_exponent(float(fin.max()) if fin.size else 0.0, fmt)
            exps[i, j] = e
            vals[i * rb:(i + 1) * rb, j * 128:(j + 1) * 128] = round8(b * 2.0 ** -e, fmt) * 2.0 ** e
    return vals, exps


def operand_values(op):
    """(values, exponents per row and block) that an Fp8Operand's buffers hold."""
    pitch = (op.k + 15) // 16 * 16
    codes = op.codes.cpu()[:op.rows * pitch].reshape(op.rows, pitch)
    assert bool((codes[:, op.k:] == 0).all()), "padding codes must be zero"
    dt = torch.float8_e4m3fn if op.fmt == 0 else torch.float8_e5m2
    v = codes[:, :op.k].contiguous().view(dt).float().numpy().astype(np.float64)
    groups = (op.k + 511) // 512
    sc = op.scales.cpu().numpy()
    row = np.arange(op.rows)[:, None]
    blk = np.arange((op.k + 127) // 128)[None, :]
    at = ((row // 128) * groups + blk // 4) * 512 + 16 * (row % 32) + 4 * ((row % 128) // 32) + blk % 4
    e = sc[at].astype(np.int64) - 127
    return v * 2.0 ** np.repeat(e, 128, axis=1)[:, :op.k].astype(np.float64), e
