"""Capturable layers under activation checkpointing, on the device's own backward thread."""
import pytest
import torch
import torch.utils.checkpoint

from paper_2312_06881_amd import nn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("reentrant", [False, True])
def test_checkpointed_capturable_layers_are_refused(reentrant):
    join = nn.AddNorm(48, p=0.4, capturable=True, device="cuda", dtype=torch.float32)
    x = torch.randn(30, 48, device="cuda", requires_grad=True)
    y = torch.randn(30, 48, device="cuda", requires_grad=True)

    def layer(x, y):
        return join(x, y)[1]

    z = torch.utils.checkpoint.checkpoint(layer, x, y, use_reentrant=reentrant)
    with pytest.raises(RuntimeError, match="capturable"):
        z.sum().backward()
    layer(x, y).sum().backward()
    assert int(join.dropout.calls) == 2 and torch.isfinite(x.grad).all()
