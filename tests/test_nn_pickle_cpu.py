"""Modules unpickled from before they had checkpoints run as they did."""
import pytest
import torch

from paper_2312_06881_amd.nn import DyadFF, DyadLinear


@pytest.mark.parametrize("make", [lambda: DyadLinear(64, 64, 4), lambda: DyadFF(64, 256, 4)], ids=["linear", "ff"])
def test_modules_without_a_stash_attribute(make):
    m = make()
    for mod in m.modules():
        del mod.__dict__["stash"]
    assert m.stash is None
    with pytest.raises(ValueError, match="device tensors"):      # that is, it reaches the library
        m(torch.zeros(5, 64, dtype=torch.bfloat16))
