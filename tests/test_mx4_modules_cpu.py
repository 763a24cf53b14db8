"""The fp4 modules outside plain inference, the C calls replaced by a product that any device can do."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2312_06881_amd import mx
from paper_2312_06881_amd.nn import DyadFF, DyadLinear, MX4DyadFF, MX4DyadLinear

calls = []


@pytest.fixture(autouse=True)
def stand_in(monkeypatch):
    def quantize_weights(w1, w2, variant="IT", n_in=None, n_out=None):
        return mx.MX4Weights(torch.zeros(64, dtype=torch.uint8), variant, n_in, n_out, w1.shape[0])

    def forward(x, weights, bias=None, act="none", workspace=None):
        calls.append(weights)
        y = torch.empty((x.shape[0], weights.n_out), dtype=x.dtype)
        y.copy_(x.detach()[:, :1] * 2.0)      # written from outside autograd's sight
        return y

    calls.clear()
    monkeypatch.setattr(mx, "quantize_weights", quantize_weights)
    monkeypatch.setattr(mx, "forward", forward)


def modules():
    torch.manual_seed(0)
    return MX4DyadLinear(DyadLinear(32, 32, 4), "gelu"), MX4DyadFF(DyadFF(32, 64, 4, ("OT", "DT")))


@pytest.mark.parametrize("which", [0, 1], ids=["linear", "ff"])
def test_a_gradient_is_refused_not_dropped(which):
    m = modules()[which]
    x = torch.randn(2, 5, 32).bfloat16().requires_grad_(True)
    y = m(x)                                        # inference on what a trainable layer made still runs
    assert y.shape == x.shape and y.requires_grad
    with pytest.raises(NotImplementedError, match="gradient"):
        (x + y).float().sum().backward()
    with torch.no_grad():
        z = m(x)
    assert torch.equal(z, y) and not z.requires_grad
    assert not m(x.detach()).requires_grad
    with torch.inference_mode():
        assert torch.equal(m(x), z)


@pytest.mark.parametrize("which", [0, 1], ids=["linear", "ff"])
def test_a_tangent_is_refused_not_dropped(which):
    m, x = modules()[which], torch.randn(5, 32).bfloat16()
    for grad in (True, False):
        with torch.set_grad_enabled(grad), forward_ad.dual_level():
            with pytest.raises(NotImplementedError, match="gradient"):
                m(forward_ad.make_dual(x, torch.ones_like(x)))
    for transform in (torch.func.vmap, torch.func.grad):
        with pytest.raises(RuntimeError):
            transform(lambda t: m(t.expand(5, 32)).float().sum())(x)


@pytest.mark.parametrize("which", [0, 1], ids=["linear", "ff"])
def test_a_trace_runs_the_product(which):
    m, x = modules()[which], torch.randn(5, 32).bfloat16()
    for grad in (True, False):
        with torch.set_grad_enabled(grad):
            traced = torch.jit.trace(m, x, check_trace=False)
            other = torch.randn(5, 32).bfloat16()
            calls.clear()
            got = traced(other)
            assert len(calls) == 1 + which
            assert torch.equal(got, m(other))
