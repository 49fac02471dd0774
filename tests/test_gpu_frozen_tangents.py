"""A frozen layer computes no derivatives in either mode: tangents are refused, not dropped."""
import pytest
import torch
from torch.autograd import forward_ad

pytestmark = pytest.mark.gpu


def test_frozen_layer_refuses_tangents(lgn):
    from paper_2006_08173_b200.layers import Int8Linear
    lin = Int8Linear(64, 48, device="cuda")
    lin.weight.requires_grad_(False)
    x = torch.randn(9, 64, device="cuda")
    lin.freeze()
    y = lin(x)
    with forward_ad.dual_level():
        with pytest.raises(RuntimeError):
            lin(forward_ad.make_dual(x, torch.ones_like(x)))
        with torch.no_grad(), pytest.raises(RuntimeError):
            lin(forward_ad.make_dual(x, torch.ones_like(x)))
        assert torch.equal(lin(x), y)                              # no tangent: as outside
    lin.freeze(False)
    with forward_ad.dual_level():
        with pytest.raises(RuntimeError):
            lin(forward_ad.make_dual(x, torch.ones_like(x)))
    assert torch.equal(lin(x), y)
