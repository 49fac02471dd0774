"""CPU-only checks of the training operators' C entries: sizes, and arguments refused before anything is enqueued."""
import ctypes as C

import pytest

P = 0x10000                                            # stands for a device address; never dereferenced on the host


def test_fp8_sizes(lgn):
    raw = lgn.raw()
    assert raw.lgn_fp8_codes_bytes(3, 17) == 3 * 32 and raw.lgn_fp8_codes_bytes(0, 5) == 0
    assert raw.lgn_fp8_scales_bytes(128, 512) == 512 and raw.lgn_fp8_scales_bytes(129, 513) == 2048
    assert raw.lgn_fp8_codes_bytes(2 ** 30 + 1, 1) == 0 and raw.lgn_fp8_scales_bytes(1, 2 ** 30 + 1) == 0
    for rows, k in ((1, 1), (5, 16), (300, 1000), (128, 512), (129, 513)):
        assert lgn._fp8_bytes(rows, k) == (raw.lgn_fp8_codes_bytes(rows, k), raw.lgn_fp8_scales_bytes(rows, k))


def test_empty_calls_do_nothing(lgn):
    raw = lgn.raw()
    assert raw.lgn_fp8_quantize(None, 0, 128, 128, 0, 0, 0, None, None, None, None, None) == 0
    assert raw.lgn_fp8_matmul(None, None, 0, None, None, 0, 0, 5, 128, None, 5, 0, 0, None, None) == 0
    assert raw.lgn_embedding(None, 10, 16, 16, 0, None, 64, 0, 1.0, None, 16, 0, None, None) == 0
    assert raw.lgn_embedding_grad(None, 16, 0, None, 64, 0, 0, 16, 1.0, -1, None, 16, 0, 0, None, 0, None) == 0


@pytest.mark.parametrize("change,code", [
    (dict(dt=2), 1), (dict(fmt=2), 1), (dict(block=2), 1), (dict(ld=255), 1), (dict(x=None), 1), (dict(x=P + 2), 1),
    (dict(codes=None), 1), (dict(scales=None), 1), (dict(codes=4 * P + 8), 1), (dict(scales=8 * P + 4), 1), (dict(codes=P), 1),
    (dict(codes=None, scales=None), 1), (dict(codes_t=16 * P), 1), (dict(rows=2 ** 31), 2), (dict(cols=2 ** 31, ld=2 ** 31), 2)])
def test_fp8_quantize_refuses(lgn, change, code):
    a = dict(x=P, rows=4, cols=256, ld=256, dt=0, fmt=0, block=0, codes=4 * P, scales=8 * P, codes_t=None, scales_t=None, stream=None)
    a.update(change)
    assert lgn.raw().lgn_fp8_quantize(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(fa=2), 1), (dict(fb=-1), 1), (dict(od=3), 1), (dict(ldo=3), 1), (dict(out=None), 1), (dict(out=16 * P + 2), 1),
    (dict(a=None), 1), (dict(sb=None), 1), (dict(a=P + 8), 1), (dict(sa=2 * P + 8), 1), (dict(status=P + 2), 1), (dict(out=P), 1),
    (dict(out=4 * P), 1), (dict(m=2 ** 31), 2), (dict(k=2 ** 31), 2)])
def test_fp8_matmul_refuses(lgn, change, code):
    a = dict(a=P, sa=2 * P, fa=0, b=4 * P, sb=6 * P, fb=0, m=4, n=4, k=256, out=16 * P, ldo=4, od=0, acc=0, status=None, stream=None)
    a.update(change)
    assert lgn.raw().lgn_fp8_matmul(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(tdt=2), 1), (dict(odt=-1), 1), (dict(bits=16), 1), (dict(ldt=15), 1), (dict(ldo=15), 1), (dict(table=None), 1), (dict(ids=None), 1),
    (dict(out=None), 1), (dict(table=P + 2), 1), (dict(ids=2 * P + 4), 1), (dict(out=P), 1), (dict(out=2 * P), 1), (dict(outside=P + 4), 1),
    (dict(vocab=2 ** 31), 2), (dict(tokens=2 ** 31), 2)])
def test_embedding_refuses(lgn, change, code):
    a = dict(table=P, vocab=10, dim=16, ldt=16, tdt=0, ids=2 * P, bits=64, tokens=4, scale=1.0, out=4 * P, ldo=16, odt=0, outside=None, stream=None)
    a.update(change)
    assert lgn.raw().lgn_embedding(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(ddt=2), 1), (dict(tdt=2), 1), (dict(bits=8), 1), (dict(ldd=15), 1), (dict(ldt=15), 1), (dict(dout=None), 1), (dict(ids=None), 1),
    (dict(table=None), 1), (dict(ws=None), 1), (dict(ws=8 * P + 8), 1), (dict(ws_bytes=100), 3), (dict(table=P), 1), (dict(ws=P), 1),
    (dict(ws=4 * P), 1), (dict(vocab=2 ** 31), 2), (dict(tokens=2 ** 31), 2)])
def test_embedding_grad_refuses(lgn, change, code):
    a = dict(dout=P, ldd=16, ddt=0, ids=2 * P, bits=64, tokens=4, vocab=10, dim=16, scale=1.0, pad=-1, table=4 * P, ldt=16, tdt=0, acc=0,
             ws=8 * P, ws_bytes=1 << 20, stream=None)
    a.update(change)
    assert lgn.raw().lgn_embedding_grad(*a.values()) == code


def test_clip_refuses(lgn):
    raw = lgn.raw()
    ws = raw.lgn_clip_workspace_bytes(1)
    assert raw.lgn_clip_workspace_bytes(0) == ws > 0 and raw.lgn_clip_workspace_bytes(513) > ws and raw.lgn_clip_workspace_bytes(-1) == 0

    def one(g=P, out=4 * P, n=100, dt=0, reserved=0):
        arr = (lgn.GradT * 1)()
        arr[0] = lgn.GradT(g, out, n, dt, reserved)
        return arr
    cases = [(one(g=None), 1), (one(out=None), 1), (one(g=P + 2), 1), (one(out=4 * P + 1), 1), (one(dt=5), 1), (one(reserved=1), 1),
             (one(out=P + 16), 1), (one(n=2 ** 41), 2)]
    for arr, code in cases:
        assert raw.lgn_clip_grad_norm(arr, 1, 1.0, 8 * P, 16 * P, ws, None) == code
        assert raw.lgn_clip_apply(arr, 1, 1.0, 8 * P, None) == code
    for max_norm in (-1.0, float("nan")):
        assert raw.lgn_clip_grad_norm(one(), 1, max_norm, 8 * P, 16 * P, ws, None) == 1
        assert raw.lgn_clip_apply(one(), 1, max_norm, 8 * P, None) == 1
    assert raw.lgn_clip_grad_norm(one(), 1, 1.0, None, 16 * P, ws, None) == 1
    assert raw.lgn_clip_grad_norm(one(), 1, 1.0, 8 * P + 4, 16 * P, ws, None) == 1
    assert raw.lgn_clip_grad_norm(one(), 1, 1.0, 8 * P, 16 * P + 8, ws, None) == 1
    assert raw.lgn_clip_grad_norm(one(), 1, 1.0, 8 * P, 16 * P, ws - 1, None) == 3
    assert raw.lgn_clip_grad_norm(None, 1, 1.0, 8 * P, 16 * P, ws, None) == 1
    assert raw.lgn_clip_grad_norm(one(), -1, 1.0, 8 * P, 16 * P, ws, None) == 1
    assert raw.lgn_grad_norm(one(out=None), -1, 8 * P, 16 * P, ws, None) == 1


def test_struct_sizes(lgn):
    assert C.sizeof(lgn.GradT) == 32 and C.sizeof(lgn.NormT) == 24
