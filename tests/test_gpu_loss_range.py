"""The loss's gradients at the ends of what their operands may hold and be long."""
import pytest
import torch

from tests.test_gpu_loss import DTYPES, check, make

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
