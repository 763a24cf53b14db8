"""Capturable dropout counts its calls on the device, which a layer that is run again for its gradient cannot."""
import pytest
import torch
import torch.utils.checkpoint

from paper_2312_06881_amd import nn


@pytest.mark.parametrize("reentrant", [False, True])
def test_checkpointed_capturable_layers_are_refused(reentrant):
    d = nn.Dropout(0.5, capturable=True)
    x = torch.ones(4, requires_grad=True)

    def layer(x):                     # its gradient is the mask's: one more than the offset here
        return x * (d.next_offset() + 1)

    y = torch.utils.checkpoint.checkpoint(layer, x, use_reentrant=reentrant)
    with pytest.raises(RuntimeError, match="capturable"):
        y.sum().backward()
    assert int(d.calls) == 1


def test_capturable_layers_elsewhere_are_not():
    d = nn.Dropout(0.5, capturable=True)
    x = torch.ones(4, requires_grad=True)
    for k in range(3):
        y = x * (d.next_offset() + 1)
        g, = torch.autograd.grad(y.sum(), x)
        assert torch.equal(g, torch.full((4,), k + 1.0))
    # another layer's checkpoint beside it, and one whose offsets come from the host
    e = nn.Dropout(0.5)
    y = torch.utils.checkpoint.checkpoint(lambda x: x * (e.next_offset() % 1000), x * (d.next_offset() + 1), use_reentrant=False)
    g, = torch.autograd.grad(y.sum(), x)
    assert torch.equal(g, torch.full((4,), 4.0 * (e.offset % 1000)))
