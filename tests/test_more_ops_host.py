"""CPU-only checks of the C entries for 8-bit integers, grouped products and distillation: sizes, and arguments refused before anything is
enqueued."""
import pytest
import torch

P = 0x10000                                            # stands for a device address; never dereferenced on the host


def test_sizes(lgn):
    raw = lgn.raw()
    assert raw.lgn_int8_codes_bytes(3, 17) == 3 * 32 and raw.lgn_int8_codes_bytes(0, 5) == 0 and raw.lgn_int8_codes_bytes(2 ** 30 + 1, 1) == 0


def test_empty_calls_do_nothing(lgn):
    raw = lgn.raw()
    assert raw.lgn_int8_quantize(None, 0, 128, 128, 0, None, None, None) == 0
    assert raw.lgn_int8_matmul(None, None, None, None, None, 32, 1, 0, 5, 128, None, 5, 0, 0, None, None) == 0
    assert raw.lgn_grouped_matmul(None, 8, None, 8, 64, 0, None, 32, 2, 0, 8, 8, None, 8, 0, 0, None, None) == 0
    assert raw.lgn_grouped_matmul(None, 8, None, 8, 64, 0, None, 32, 2, 4, 0, 8, None, 8, 0, 0, None, None) == 0
    assert raw.lgn_grouped_weight_grad(None, 8, None, 8, None, 32, 2, 4, 0, 8, None, 8, 64, 0, 0, None, None) == 0
    assert raw.lgn_distill_loss(None, 0, 10, 10, 0, None, 32, 4, None, 4, 0, 4, None, 32, 1.0, 1.0, None, None, None, 10, None) == 0


@pytest.mark.parametrize("change,code", [
    (dict(dt=2), 1), (dict(ld=255), 1), (dict(x=None), 1), (dict(x=P + 2), 1), (dict(codes=None), 1), (dict(scales=None), 1), (dict(codes=4 * P + 8), 1),
    (dict(scales=8 * P + 2), 1), (dict(codes=P), 1), (dict(scales=4 * P), 1), (dict(scales=P + 64), 1), (dict(rows=2 ** 31), 2), (dict(cols=2 ** 31, ld=2 ** 31), 2),
    (dict(ld=2 ** 41), 1)])
def test_int8_quantize_refuses(lgn, change, code):
    a = dict(x=P, rows=4, cols=256, ld=256, dt=0, codes=4 * P, scales=8 * P, stream=None)
    a.update(change)
    assert lgn.raw().lgn_int8_quantize(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(od=3), 1), (dict(bits=16), 1), (dict(groups=0), 1), (dict(groups=2), 1), (dict(ldo=3), 1), (dict(out=None), 1), (dict(out=16 * P + 2), 1), (dict(a=None), 1),
    (dict(sb=None), 1), (dict(sa=None), 1), (dict(b=4 * P + 8), 1), (dict(sa=2 * P + 2), 1), (dict(status=P + 2), 1), (dict(out=P), 1), (dict(out=4 * P), 1), (dict(out=6 * P), 1),
    (dict(offsets=16 * P, groups=2), 1), (dict(offsets=9 * P + 2, groups=2), 1), (dict(m=2 ** 31), 2), (dict(k=2 ** 17 + 1), 2), (dict(offsets=9 * P, groups=2 ** 21), 2),
    (dict(offsets=9 * P, groups=2 ** 20, n=2 ** 11, ldo=2 ** 11), 2)])
def test_int8_matmul_refuses(lgn, change, code):
    a = dict(a=P, sa=2 * P, b=4 * P, sb=6 * P, offsets=None, bits=32, groups=1, m=4, n=4, k=256, out=16 * P, ldo=4, od=0, rest=0, status=None, stream=None)
    a.update(change)
    assert lgn.raw().lgn_int8_matmul(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(od=2), 1), (dict(bits=8), 1), (dict(groups=0), 1), (dict(offsets=None), 1), (dict(offsets=9 * P + 4), 1), (dict(ldo=7), 1), (dict(out=None), 1), (dict(out=16 * P + 2), 1),
    (dict(x=None), 1), (dict(w=None), 1), (dict(x=P + 8), 1), (dict(w=4 * P + 2), 1), (dict(ldx=65), 1), (dict(ldx=56), 1), (dict(ldw=68), 1), (dict(w_group=8 * 64 + 4), 1),
    (dict(w_group=8 * 64 - 8), 1), (dict(out=P), 1), (dict(out=4 * P + 1024), 1), (dict(out=9 * P - 64), 1), (dict(status=P + 2), 1), (dict(rows=2 ** 31), 2), (dict(k=2 ** 31), 2),
    (dict(n=2 ** 31), 2), (dict(groups=2 ** 21), 2)])
def test_grouped_matmul_refuses(lgn, change, code):
    a = dict(x=P, ldx=64, w=4 * P, ldw=64, w_group=8 * 64, transposed=0, offsets=9 * P, bits=64, groups=3, rows=5, n=8, k=64, out=16 * P, ldo=8, od=0, rest=0, status=None, stream=None)
    a.update(change)
    assert lgn.raw().lgn_grouped_matmul(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(od=2), 1), (dict(bits=8), 1), (dict(groups=0), 1), (dict(offsets=None), 1), (dict(ldo=7), 1), (dict(out=None), 1), (dict(out=16 * P + 1), 1), (dict(dy=None), 1), (dict(x=None), 1),
    (dict(dy=P + 8), 1), (dict(lddy=17), 1), (dict(ldx=4), 1), (dict(group=16 * 8 - 1), 1), (dict(out=P), 1), (dict(out=4 * P), 1), (dict(out=9 * P - 64), 1), (dict(status=P + 2), 1),
    (dict(rows=2 ** 31), 2), (dict(m=2 ** 31), 2), (dict(n=2 ** 31), 2)])
def test_weight_grad_refuses(lgn, change, code):
    a = dict(dy=P, lddy=16, x=4 * P, ldx=8, offsets=9 * P, bits=32, groups=3, rows=5, m=16, n=8, out=16 * P, ldo=8, group=16 * 8, od=0, acc=0, status=None, stream=None)
    a.update(change)
    assert lgn.raw().lgn_grouped_weight_grad(*a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(dt=2), 1), (dict(tdt=2), 1), (dict(bits=16), 1), (dict(lbits=8), 1), (dict(T=0.0), 1), (dict(T=float("nan")), 1), (dict(T=-1.0), 1), (dict(T=1e4), 1), (dict(alpha=-0.1), 1), (dict(alpha=1.1), 1),
    (dict(alpha=float("nan")), 1), (dict(logits=None), 1), (dict(logits=P + 2), 1), (dict(ld=99), 1), (dict(ids=None), 1), (dict(teacher=None), 1), (dict(ids=3 * P + 4), 1), (dict(teacher=4 * P + 2), 1),
    (dict(ld_ids=4), 1), (dict(ld_t=4), 1), (dict(labels=5 * P + 4), 1), (dict(weight=6 * P + 2), 1), (dict(loss=None), 1), (dict(loss=7 * P + 2), 1), (dict(dl=8 * P + 2), 1), (dict(ldd=99), 1),
    (dict(dl=P + 16), 1), (dict(dl=P, ldd=104), 1), (dict(dl=3 * P), 1), (dict(dl=4 * P), 1), (dict(dl=6 * P), 1), (dict(dl=7 * P), 1), (dict(loss=P), 1), (dict(loss=6 * P), 1),
    (dict(tokens=2 ** 31), 2), (dict(vocab=2 ** 31, ld=2 ** 31), 2), (dict(top=1025, ld_ids=1025, ld_t=1025), 2)])
def test_distill_refuses(lgn, change, code):
    a = dict(logits=P, tokens=4, vocab=100, ld=100, dt=0, ids=3 * P, bits=64, ld_ids=5, teacher=4 * P, ld_t=5, tdt=0, top=5, labels=5 * P, lbits=64, T=1.0, alpha=0.5, weight=6 * P, loss=7 * P,
             dl=8 * P, ldd=100, stream=None)
    a.update(change)
    assert lgn.raw().lgn_distill_loss(*a.values()) == code


def test_selftest_refuses(lgn):
    raw = lgn.raw()
    assert raw.lgn_selftest_grouped_wait_expires(P, 4 * P, 0, 9 * P, 32, 2, 8, 8, 8, 16 * P, 0, None, None) == 1
    assert raw.lgn_selftest_grouped_wait_expires(P, 4 * P, 0, 9 * P, 32, 2, 0, 8, 8, 16 * P, 0, 12 * P, None) == 1


class Stand:
    """A contiguous CUDA tensor as far as the binding looks at one."""
    is_cuda = True

    def __init__(self, *shape, dtype=torch.float32, at=0):
        self.shape, self.dtype, self.at = torch.Size(shape), dtype, at

    device = property(lambda self: torch.device("cuda", self.at))
    get_device = lambda self: self.at
    data_ptr = lambda self: 0x10000
    is_contiguous = lambda self: True
    element_size = lambda self: self.dtype.itemsize
    stride = lambda self: tuple(int(torch.Size(self.shape[i + 1:]).numel()) for i in range(len(self.shape)))
    numel = lambda self: int(self.shape.numel())
    dim = lambda self: len(self.shape)
    size = lambda self, d: self.shape[d]


def stand_int8(lgn, rows, k, at=0):
    return lgn.Int8Operand(Stand(rows, (k + 15) // 16 * 16, dtype=torch.int8, at=at), Stand(rows, at=at), rows, k)


def test_binding_refuses(lgn, monkeypatch):
    monkeypatch.setattr(lgn, "_current_device", lambda: 0)
    bf, i64 = torch.bfloat16, torch.int64
    x, w, off, dy = Stand(5, 64, dtype=bf), Stand(2, 8, 64, dtype=bf), Stand(3, dtype=i64), Stand(5, 8, dtype=bf)
    with pytest.raises(ValueError):
        stand_int8(lgn, 4, 64)._codes and lgn.Int8Operand(Stand(3, 64, dtype=torch.int8), Stand(4), 4, 64)
    for bad in (lambda: lgn.Int8Operand(Stand(4, 64), Stand(4), 4, 64), lambda: lgn.lgn_grouped_matmul(Stand(5, 64), w, off), lambda: lgn.lgn_grouped_matmul(x, w, Stand(3)),
                lambda: lgn.lgn_distill_loss(Stand(4, 9), Stand(4, 2, dtype=i64), Stand(4, 2), weight=Stand(4, dtype=bf)),
                lambda: lgn.lgn_distill_loss(Stand(4, 9), Stand(4, 2), Stand(4, 2)), lambda: lgn.lgn_distill_loss(Stand(4, 9), Stand(4, 2, dtype=i64), Stand(4, 2), dlogits=Stand(4, 9, dtype=bf))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: lgn.lgn_int8_matmul(stand_int8(lgn, 4, 64), stand_int8(lgn, 4, 80)), lambda: lgn.lgn_int8_matmul(stand_int8(lgn, 4, 64), stand_int8(lgn, 5, 64), offsets=off),
                lambda: lgn.lgn_int8_matmul(stand_int8(lgn, 4, 64), stand_int8(lgn, 4, 64), out=Stand(4, 5)), lambda: lgn.lgn_int8_quantize(Stand(4, 64), out=stand_int8(lgn, 4, 65)),
                lambda: lgn.lgn_grouped_matmul(x, Stand(3, 8, 64, dtype=bf), off), lambda: lgn.lgn_grouped_matmul(x, Stand(2, 8, 63, dtype=bf), off),
                lambda: lgn.lgn_grouped_matmul(x, w, off, transposed=True), lambda: lgn.lgn_grouped_matmul(x, w, off, out=Stand(5, 9)), lambda: lgn.lgn_grouped_matmul(x, w, Stand(1, dtype=i64)),
                lambda: lgn.lgn_grouped_weight_grad(dy, Stand(6, 64, dtype=bf), off), lambda: lgn.lgn_grouped_weight_grad(dy, x, off, accumulate=True),
                lambda: lgn.lgn_grouped_weight_grad(dy, x, off, out=Stand(2, 64, 8)), lambda: lgn.lgn_distill_loss(Stand(4, 9), Stand(3, 2, dtype=i64), Stand(4, 2)),
                lambda: lgn.lgn_distill_loss(Stand(4, 9), Stand(4, 2, dtype=i64), Stand(4, 3)), lambda: lgn.lgn_distill_loss(Stand(4, 9), Stand(4, 2, dtype=i64), Stand(4, 2), labels=Stand(5, dtype=i64)),
                lambda: lgn.lgn_distill_loss(Stand(4, 9), Stand(4, 2, dtype=i64), Stand(4, 2), dlogits=Stand(4, 8)),
                lambda: lgn.lgn_distill_loss(torch.zeros(4, 9), Stand(4, 2, dtype=i64), Stand(4, 2))):
        with pytest.raises(ValueError):
            bad()


def test_several_devices_are_refused(lgn, monkeypatch):
    monkeypatch.setattr(lgn, "_current_device", lambda: 0)
    bf, i64 = torch.bfloat16, torch.int64
    x, w, off, dy = Stand(5, 64, dtype=bf), Stand(2, 8, 64, dtype=bf), Stand(3, dtype=i64), Stand(5, 8, dtype=bf)
    far = Stand(3, dtype=i64, at=1)
    for bad in (lambda: lgn.lgn_int8_matmul(stand_int8(lgn, 4, 64), stand_int8(lgn, 4, 64, 1)), lambda: lgn.lgn_int8_matmul(stand_int8(lgn, 4, 64), stand_int8(lgn, 4, 64), offsets=far),
                lambda: lgn.lgn_int8_quantize(Stand(4, 64), out=stand_int8(lgn, 4, 64, 1)), lambda: lgn.lgn_grouped_matmul(x, w, far), lambda: lgn.lgn_grouped_matmul(x, Stand(2, 8, 64, dtype=bf, at=1), off),
                lambda: lgn.lgn_grouped_weight_grad(dy, x, far), lambda: lgn.lgn_grouped_weight_grad(Stand(5, 8, dtype=bf, at=1), x, off),
                lambda: lgn.lgn_distill_loss(Stand(4, 9), Stand(4, 2, dtype=i64, at=1), Stand(4, 2)), lambda: lgn.lgn_distill_loss(Stand(4, 9), Stand(4, 2, dtype=i64), Stand(4, 2), weight=Stand(4, at=1))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ValueError):
        lgn.Int8Operand(Stand(4, 64, dtype=torch.int8), Stand(4, at=1), 4, 64)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), 1), (dict(x=P + 1), 1), (dict(ld=9), 1), (dict(ld=2 ** 41), 1), (dict(group=2 ** 41), 1), (dict(out=None), 1), (dict(out=64 * P + 8), 1), (dict(out=P), 1), (dict(rows=2 ** 31), 2),
    (dict(cols=2 ** 31, ld=2 ** 31), 2), (dict(groups=2 ** 21), 2), (dict(rows=0, x=None, out=None), 0)])
def test_align_rows_refuses(lgn, change, code):
    a = dict(x=P, ld=10, group=50, groups=3, rows=5, cols=10, out=64 * P, stream=None)
    a.update(change)
    assert lgn.raw().lgn_align_rows(*a.values()) == code


def test_distill_loss_of_other_rows_is_refused(lgn):
    """As many values in another order would be other rows' values."""
    from paper_2006_08173_b200.layers import DistillLoss
    s, ids, z, labels = torch.zeros(2, 3, 50), torch.zeros(2, 3, 4, dtype=torch.int64), torch.zeros(2, 3, 4), torch.zeros(2, 3, dtype=torch.int64)
    for bad in ((s, ids.reshape(3, 2, 4), z), (s, ids, z.reshape(3, 2, 4)), (s, ids, z.reshape(2, 6, 2)), (s, ids, z, labels.reshape(3, 2)), (s, ids, z, labels.reshape(6))):
        with pytest.raises(ValueError, match="same rows"):
            DistillLoss()(*bad)


@pytest.mark.parametrize("dtype", [torch.uint8, torch.int8, torch.int16, torch.int32, torch.int64])
@pytest.mark.parametrize("experts", [1, 5, 127, 128, 256])
def test_by_expert(lgn, dtype, experts):
    from paper_2006_08173_b200.layers import by_expert
    top = min(experts, torch.iinfo(dtype).max)
    ids = torch.arange(500).mul(7919).remainder(top + 1).to(dtype)
    order, offsets = by_expert(ids, experts)
    ends = offsets.tolist()
    assert len(ends) == experts + 1 and sorted(order.tolist()) == list(range(500))
    for e in range(experts):
        assert order[ends[e]:ends[e + 1]].tolist() == [i for i in range(500) if int(ids[i]) == e]
    assert by_expert(ids[:0], experts)[1].tolist() == [0] * (experts + 1)
