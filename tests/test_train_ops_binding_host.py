"""CPU-only: arguments that the binding refuses before it calls the library."""
import pytest
import torch


@pytest.fixture
def no_calls(lgn, monkeypatch):
    class Library:
        def __getattr__(self, name):
            def call(*args):
                raise AssertionError(f"{name} was called")
            return call
    monkeypatch.setattr(lgn, "_lib", Library())
    monkeypatch.setattr(lgn, "_current_device", lambda: 0)
    monkeypatch.setattr(lgn, "_raw_stream", lambda device: 0)


def test_operands_in_host_memory(lgn, no_calls):
    """Their addresses would reach a kernel."""
    with pytest.raises(ValueError):
        lgn.new_fp8_operand(4, 256, lgn.E4M3, "cpu")
    with pytest.raises(ValueError):
        lgn.Fp8Operand.empty(4, 256, lgn.E5M2, torch.device("cpu"))
    with pytest.raises(ValueError):
        lgn.Fp8Operand(torch.zeros(1024, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 4, 256, lgn.E4M3)


def test_words_that_are_too_small(lgn, no_calls):
    """What the library writes one value to: 4 bytes of status, 8 of a count."""
    from test_train_ops_devices import Stand, operand
    a, out = operand(lgn, 0), Stand(0, 4, 4)
    for word in (Stand(0, 0, dtype=torch.int32), Stand(0, 1, dtype=torch.uint8), Stand(0, 3, dtype=torch.uint8), Stand(0, 1, dtype=torch.int16)):
        with pytest.raises(ValueError):
            lgn.lgn_fp8_matmul(a, a, out=out, status=word)
        with pytest.raises(ValueError):
            lgn.lgn_selftest_matmul_wait_expires(a, a, out, word)
    with pytest.raises(ValueError):
        lgn.lgn_embedding(Stand(0, 10, 16), Stand(0, 4, dtype=torch.int64), out=Stand(0, 4, 16), n_outside=Stand(0, 0, dtype=torch.int64))


def test_tensors_that_are_written_over_one_another(lgn, no_calls):
    """The same gradient twice, or an out over another tensor: refused where something is written, not for the norm alone."""
    from test_train_ops_devices import Stand

    def at(address, n, dtype=torch.float32):
        t = Stand(0, n, dtype=dtype)
        t.data_ptr = lambda: address
        return t
    rec, ws = Stand(0, 24, dtype=torch.uint8), Stand(0, 4096, dtype=torch.uint8)
    a, b, c = at(0x1000, 100), at(0x2000, 100), at(0x3000, 1000, torch.bfloat16)
    bad = [([a, a], None), ([a, b, a], None), ([a, b], [at(0x3000, 100), at(0x3004, 100)]), ([a, b], [b, a]), ([a, b], [a, at(0x1000 + 396, 100)]),
           ([a, at(0x1000 + 40, 10)], None), ([c, b], [at(0x2000 - 1996, 1000, torch.bfloat16), at(0x9000, 100)]), ([a, a], [b, b])]
    for grads, outs in bad:
        g = lgn.make_grads(grads, outs)
        with pytest.raises(ValueError):
            lgn.lgn_clip_grad_norm(g, 1.0, rec, ws)
        with pytest.raises(ValueError):
            lgn.lgn_clip_apply(g, 1.0, rec)
        with pytest.raises(AssertionError, match="lgn_grad_norm was called"):
            lgn.lgn_grad_norm(g, rec, ws)
    good = [([a, b, c], None), ([a, a], [b, at(0x9000, 100)]), ([a, b], [a, at(0x9000, 100)]), ([a, at(0x1000, 0), at(0x1000 + 400, 5)], None),
            ([a, at(0x1000 + 40, 10)], [b, at(0x9000, 10)]), ([], None)]
    for grads, outs in good:
        with pytest.raises(AssertionError, match="lgn_clip_grad_norm was called"):
            lgn.lgn_clip_grad_norm(lgn.make_grads(grads, outs), 1.0, rec, ws)
