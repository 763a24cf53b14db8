"""The loss's gradients at the ends of what their operands may hold and be long."""
import pytest
import torch

from paper_2312_06881_amd import nn
from tests.test_gpu_loss import BF, DTYPES, F, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("top", [2.0 ** 112, 2.0 ** 116, 2.0 ** 122])
@pytest.mark.parametrize("M", [50, 300])
def test_columns_of_the_largest_magnitudes(M, top, dtype):
    # a column of W, or of X, near the type's end beside one of zeros, so that the logits do not have it
    x, w, t = make(M, 64, 300, dtype)
    x[:, 9] = 0.0
    w[:, 9] *= top
    w[:, 17] = 0.0
    x[:, 17] *= top
    _, dx, dw = check(x, w, t, "sum")
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()


def test_long_vocabularies_keep_their_small_terms():
    # Every token's target is entry 0, whose row is 1; the other rows are c, and x is 0, so each of V entries has
    # probability 1 / V and dx = c (V - 1) / V + (1 / V - 1).  A target's term of -1 stands in the sum from its first
    # step on, and 32 of the others, what one matrix instruction adds, come to 0.9 of half of that sum's last bit: they
    # are lost wherever they meet it.  With at most 16384 entries in one sum that is at most 512 additions of 2^-25; the
    # other products of the split operands (2^-8 of these) and a handful of last additions 2^-24 stay below 16 of them.
    M, n, V = 2048, 8192, 43520
    w = torch.full((V, n), 0.9 * 2.0 ** -25 * V / 32, device="cuda", dtype=F)
    c = float(w[1, 0])
    w[0] = 1.0
    x = torch.zeros((M, n), device="cuda", dtype=F, requires_grad=True)
    loss = nn.linear_cross_entropy(x, w, torch.zeros(M, device="cuda", dtype=torch.int64), reduction="sum")
    dx, = torch.autograd.grad(loss, x)
    want = c * (V - 1) / V + (1 / V - 1)
    assert float((dx.double() - want).abs().max()) <= (512 + 16) * 2.0 ** -25


@pytest.mark.parametrize("M,n,V,dtype", [(130, 16384, 5600, F), (130, 16392, 17000, BF), (600, 5000, 20011, F)])
def test_weights_laid_out_a_piece_at_a_time(M, n, V, dtype):
    # more than 512 MB of them, in both passes
    check(*make(M, n, V, dtype))
