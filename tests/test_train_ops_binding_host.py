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


def test_operands_in_host_memory(lgn, no_calls):
    """Their addresses would reach a kernel."""
    with pytest.raises(ValueError):
        lgn.new_fp8_operand(4, 256, lgn.E4M3, "cpu")
    with pytest.raises(ValueError):
        lgn.Fp8Operand.empty(4, 256, lgn.E5M2, torch.device("cpu"))
    with pytest.raises(ValueError):
        lgn.Fp8Operand(torch.zeros(1024, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 4, 256, lgn.E4M3)


def test_words_that_are_too_small(lgn, no_calls, monkeypatch):
    """What the library writes one value to: 4 bytes of status, 8 of a count."""
    from test_train_ops_devices import Stand, operand
    monkeypatch.setattr(lgn, "_current_device", lambda: 0)
    a, out = operand(lgn, 0), Stand(0, 4, 4)
    for word in (Stand(0, 0, dtype=torch.int32), Stand(0, 1, dtype=torch.uint8), Stand(0, 3, dtype=torch.uint8), Stand(0, 1, dtype=torch.int16)):
        with pytest.raises(ValueError):
            lgn.lgn_fp8_matmul(a, a, out=out, status=word)
        with pytest.raises(ValueError):
            lgn.lgn_selftest_matmul_wait_expires(a, a, out, word)
    with pytest.raises(ValueError):
        lgn.lgn_embedding(Stand(0, 10, 16), Stand(0, 4, dtype=torch.int64), out=Stand(0, 4, 16), n_outside=Stand(0, 0, dtype=torch.int64))
