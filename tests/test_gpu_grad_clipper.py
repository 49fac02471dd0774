"""GradClipper over several steps."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers(lgn):
    from paper_2006_08173_b200 import layers as mod
    return mod


def parameters(*sizes):
    return [torch.nn.Parameter(torch.zeros(n, device="cuda")) for n in sizes]


def test_a_gradient_that_comes_later_takes_part(layers):
    """Sums of squares of small integers are exact, so the norms are the rounded square roots."""
    a, b, c = parameters(4, 9, 16)
    a.grad = torch.full((4,), 2.0, device="cuda")
    clip = layers.GradClipper([a, b, c], 1.0)
    assert float(clip.clip()) == 4.0 and bool((a.grad == 0.5).all())
    b.grad = torch.full((9,), 1.0, device="cuda")
    a.grad.fill_(2.0)
    assert float(clip.clip()) == 5.0                              # sqrt(16 + 9)
    assert bool((a.grad == torch.tensor(2.0) * torch.tensor(0.2)).all()) and bool((b.grad == torch.tensor(0.2)).all())
    c.grad = torch.full((16,), 3.0, device="cuda")
    a.grad.zero_()
    b.grad.fill_(5.0)                                             # 225 + 144 = 369
    norm = float(clip.clip())
    assert abs(norm - 369 ** 0.5) <= 2.0 ** -24 * norm
    for g, v in ((a.grad, 0.0), (b.grad, 5.0), (c.grad, 3.0)):
        assert bool(((g - v / 369 ** 0.5).abs() <= 4 * 2.0 ** -24 * v).all())
    with pytest.raises(RuntimeError):
        c.grad = torch.ones(16, device="cuda")
        clip.clip()


def test_norms_of_several_steps_are_kept(layers):
    """On the current stream, another one, and one given by its handle."""
    (p,) = parameters(4)
    p.grad = torch.zeros(4, device="cuda")
    clip = layers.GradClipper([p], 100.0)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    norms = []
    for step, stream in enumerate([None, None, other, other, other.cuda_stream, other.cuda_stream, None]):
        p.grad.fill_(float(step))
        torch.cuda.synchronize()
        norms.append(clip.clip(stream))
        torch.cuda.synchronize()
    assert [float(n) for n in norms] == [0.0, 2.0, 4.0, 6.0, 8.0, 10.0, 12.0]
