"""Fp8Linear.check(): a device-side wait that runs out in any of a layer's calls is reported, and the layer works on.  The time-outs
are the library's own self-tests, put in the place of the calls."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers(lgn):
    from paper_2006_08173_b200 import layers as mod
    return mod


def step(lin, x):
    y = lin(x)
    y.backward(torch.exp(torch.randn_like(y)))
    return y


def test_every_call_reports(lgn, layers, monkeypatch):
    lin = layers.Fp8Linear(128, 64, sparsity=0.5, device="cuda")
    lin.check()
    x = torch.randn(40, 128, device="cuda", requires_grad=True)
    seen, real = [], lgn.lgn_fp8_matmul

    def matmul(*args, **kw):
        seen.append(kw.get("status"))
        return real(*args, **kw)
    monkeypatch.setattr(lgn, "lgn_fp8_matmul", matmul)
    step(lin, x)
    assert len(seen) == 3 and all(s is not None and s is seen[0] for s in seen)
    lin.check()


def test_a_product_that_times_out(lgn, layers, monkeypatch):
    lin = layers.Fp8Linear(128, 64, device="cuda")
    x = torch.randn(40, 128, device="cuda")
    want = lin(x)

    def withheld(a, b, out_dtype, status):
        out = torch.empty(a.rows, b.rows, dtype=out_dtype, device="cuda")
        lgn.lgn_selftest_matmul_wait_expires(a, b, out, status)
        return out
    with monkeypatch.context() as m:
        m.setattr(lgn, "lgn_fp8_matmul", withheld)
        lin(x)
    lin(x)                                                         # a good pass does not clear the report
    with pytest.raises(lgn.LgnError) as e:
        lin.check()
    assert e.value.code == 5
    assert torch.equal(lin(x), want)
    lin.check()


def test_a_pruning_that_times_out(lgn, layers, monkeypatch):
    lin = layers.Fp8Linear(128, 64, sparsity=0.5, device="cuda")
    x = torch.randn(40, 128, device="cuda", requires_grad=True)
    with monkeypatch.context() as m:
        m.setattr(lgn, "lgn_compress_layers", lgn.lgn_selftest_wait_expires)
        step(lin, x)
    with pytest.raises(lgn.LgnError) as e:
        lin.check()
    assert e.value.code == 5
    step(lin, x)
    lin.check()


def test_passes_on_another_stream(lgn, layers, monkeypatch):
    """check() waits for them too."""
    lin = layers.Fp8Linear(128, 64, device="cuda")
    x = torch.randn(40, 128, device="cuda")
    lin(x)
    lin.check()

    def withheld(a, b, out_dtype, status):
        out = torch.empty(a.rows, b.rows, dtype=out_dtype, device="cuda")
        lgn.lgn_selftest_matmul_wait_expires(a, b, out, status)
        return out
    side = torch.cuda.Stream()
    with monkeypatch.context() as m, torch.cuda.stream(side):
        m.setattr(lgn, "lgn_fp8_matmul", withheld)
        lin(x)
    with pytest.raises(lgn.LgnError):
        lin.check()
    lin.check()
