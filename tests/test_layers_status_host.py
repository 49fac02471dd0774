"""CPU-only: a pass that is refused for lack of a device leaves nothing behind for check()."""
import pytest
import torch


def test_check_after_a_refused_pass(lgn):
    from paper_2006_08173_b200.layers import ExpertLinear, Fp8Linear, Int8Linear
    offsets = torch.tensor([0, 2, 3])
    for layer, args in ((Fp8Linear(64, 48), ()), (Int8Linear(64, 48), ()), (ExpertLinear(2, 64, 48), (offsets,))):
        with pytest.raises(ValueError):
            layer(torch.zeros(3, 64), *args)
        layer.check()
        assert not layer._status
