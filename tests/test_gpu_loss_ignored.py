"""Tokens that do not count leave no trace in the gradients, whatever they and the weights hold."""
import pytest
import torch

from paper_2312_06881_amd import nn
from tests.test_gpu_loss import DTYPES, make

pytestmark = pytest.mark.gpu


def gradients(x, w, t, dloss=None):
    a, b = x.cuda().requires_grad_(True), w.cuda().requires_grad_(True)
    each = nn.linear_cross_entropy(a, b, t.cuda(), reduction="none")
    return torch.autograd.grad(each, (a, b), torch.ones_like(each) if dloss is None else dloss.cuda())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [1, 70, 128, 129, 200, 256, 257, 600])
def test_what_an_ignored_token_holds_reaches_no_gradient(M, dtype):
    x, w, t = make(M, 72, 400, dtype, ignored=0.0)
    t[::5] = -100
    t[-1] = 400
    bad = x.clone()
    bad[::5, 3] = float("nan")
    bad[::10, 4] = float("inf")
    bad[-1, ::2] = -float("inf")
    for got, want in zip(gradients(bad, w, t), gradients(x, w, t)):
        assert torch.equal(got, want) and torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [1, 70, 129, 256, 600])
def test_an_ignored_token_has_no_gradient_beside_infinite_weights(M, dtype):
    x, w, t = make(M, 72, 400, dtype, ignored=0.0)
    t[::3] = -100
    w[7, 5] = float("inf")
    dx, _ = gradients(x, w, t)
    assert not dx[::3].any()
