"""CPU-only: arguments that the binding refuses before it calls the library."""
import pytest
import torch


@pytest.fixture
def no_calls(lgn, monkeypatch):
    class Library:
        def __getattr__(self, name):
            raise AssertionError(f"{name} was called")
    monkeypatch.setattr(lgn, "_lib", Library())


def test_operands_in_host_memory(lgn, no_calls):
    """Their addresses would reach a kernel."""
    with pytest.raises(ValueError):
        lgn.new_fp8_operand(4, 256, lgn.E4M3, "cpu")
    with pytest.raises(ValueError):
        lgn.Fp8Operand.empty(4, 256, lgn.E5M2, torch.device("cpu"))
    with pytest.raises(ValueError):
        lgn.Fp8Operand(torch.zeros(1024, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 4, 256, lgn.E4M3)
