"""CPU-only: calls of the training operators are made on their tensors' device, and refused where the tensors are on several.
Tensors, the library and the current device are stand-ins; what is looked at is the device that is current when the library is
called, and the stream it is given."""
import contextlib

import pytest
import torch


class Stand:
    """A contiguous CUDA tensor as far as the binding looks at one."""
    is_cuda = True

    def __init__(self, device, *shape, dtype=torch.float32):
        self.at, self.shape, self.dtype = device, tuple(shape), dtype

    device = property(lambda self: torch.device("cuda", self.at))
    get_device = lambda self: self.at
    data_ptr = lambda self: 0x10000 * (self.at + 1)
    is_contiguous = lambda self: True
    element_size = lambda self: self.dtype.itemsize
    stride = lambda self: tuple(int(torch.Size(self.shape[i + 1:]).numel()) for i in range(len(self.shape)))
    numel = lambda self: int(torch.Size(self.shape).numel())
    dim = lambda self: len(self.shape)


@pytest.fixture
def calls(lgn, monkeypatch):
    """(entry point, device current then, stream argument) of the calls made."""
    now, seen = [0], []

    @contextlib.contextmanager
    def device(index):
        before, now[0] = now[0], index
        yield
        now[0] = before

    class Library:
        def __getattr__(self, name):
            def call(*args):
                seen.append((name, now[0], args[-1]))
                return 0
            return (lambda *args: 4096) if name.endswith("_bytes") else call

    monkeypatch.setattr(lgn, "_lib", Library())
    monkeypatch.setattr(lgn, "_current_device", lambda: now[0])
    monkeypatch.setattr(lgn, "_raw_stream", lambda index: 700 + index)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch, "empty", lambda shape, dtype=None, device=None: Stand(torch.device(device).index, *((shape,) if isinstance(shape, int) else shape), dtype=dtype))
    return seen


def operand(lgn, device, rows=4, k=128):
    return lgn.Fp8Operand(Stand(device, rows * k, dtype=torch.uint8), Stand(device, 512, dtype=torch.uint8), rows, k, lgn.E4M3)


def every_call(lgn, d, e):
    """Each entry point with tensors on device d and one of them on e."""
    f, i, u8 = torch.float32, torch.int64, torch.uint8
    table, ids, flat = Stand(d, 10, 16), Stand(e, 4, dtype=i), Stand(d, 100)
    yield "quantize", lambda: lgn.lgn_fp8_quantize(Stand(d, 4, 128), out=operand(lgn, e))
    yield "quantize", lambda: lgn.lgn_fp8_quantize(Stand(d, 128, 4), rowwise=False, transposed=True, out_t=operand(lgn, e))
    yield "matmul", lambda: lgn.lgn_fp8_matmul(operand(lgn, d), operand(lgn, e))
    yield "matmul", lambda: lgn.lgn_fp8_matmul(operand(lgn, d), operand(lgn, d), out=Stand(e, 4, 4))
    yield "matmul", lambda: lgn.lgn_fp8_matmul(operand(lgn, d), operand(lgn, d), status=Stand(e, 1, dtype=torch.int32))
    yield "selftest", lambda: lgn.lgn_selftest_matmul_wait_expires(operand(lgn, d), operand(lgn, d), Stand(d, 4, 4), Stand(e, 1, dtype=torch.int32))
    yield "embedding", lambda: lgn.lgn_embedding(table, ids)
    yield "embedding", lambda: lgn.lgn_embedding(table, Stand(d, 4, dtype=i), out=Stand(e, 4, 16))
    yield "embedding", lambda: lgn.lgn_embedding(table, Stand(d, 4, dtype=i), n_outside=Stand(e, 1, dtype=i))
    yield "embedding_grad", lambda: lgn.lgn_embedding_grad(Stand(d, 4, 16), ids, 10)
    yield "embedding_grad", lambda: lgn.lgn_embedding_grad(Stand(d, 4, 16), Stand(d, 4, dtype=i), 10, ws=Stand(e, 4096, dtype=u8))
    yield "norm", lambda: lgn.lgn_grad_norm(lgn.make_grads([flat]), Stand(d, 24, dtype=u8), Stand(e, 4096, dtype=u8))
    yield "norm", lambda: lgn.lgn_grad_norm(lgn.make_grads([flat]), Stand(e, 24, dtype=u8), Stand(d, 4096, dtype=u8))
    yield "clip", lambda: lgn.lgn_clip_grad_norm(lgn.make_grads([flat], [Stand(e, 100)]), 1.0, Stand(d, 24, dtype=u8), Stand(d, 4096, dtype=u8))
    yield "clip", lambda: lgn.lgn_clip_grad_norm(lgn.make_grads([flat]), 1.0, Stand(e, 24, dtype=u8), Stand(d, 4096, dtype=u8))
    yield "apply", lambda: lgn.lgn_clip_apply(lgn.make_grads([flat]), 1.0, Stand(e, 24, dtype=u8))


@pytest.mark.parametrize("device", [0, 1])
def test_calls_are_made_on_the_tensors_device(lgn, calls, device):
    n = 0
    for what, call in every_call(lgn, device, device):
        call()
        n += 1
        assert len(calls) == n and what in calls[-1][0] and calls[-1][1:] == (device, 700 + device)
    assert lgn._current_device() == 0


def test_tensors_on_several_devices_are_refused(lgn, calls):
    for d, e in ((0, 1), (1, 0)):
        for what, call in every_call(lgn, d, e):
            with pytest.raises(ValueError):
                call()
    with pytest.raises(ValueError):
        lgn.Fp8Operand(Stand(0, 512, dtype=torch.uint8), Stand(1, 512, dtype=torch.uint8), 4, 128, lgn.E4M3)
    assert calls == []


def test_a_stream_of_another_device_is_refused(lgn, calls, monkeypatch):
    class Stream:
        device_index, cuda_stream = 1, 5

    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    with pytest.raises(ValueError):
        lgn.lgn_fp8_quantize(Stand(0, 4, 128), out=operand(lgn, 0), stream=Stream())
    lgn.lgn_fp8_quantize(Stand(1, 4, 128), out=operand(lgn, 1), stream=Stream())
    assert calls == [("lgn_fp8_quantize", 1, 5)]
