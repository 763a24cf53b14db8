"""Where the dropout layers draw their seeds and offsets, without a GPU."""
import pytest
import torch

from paper_2312_06881_amd import nn


@pytest.mark.parametrize("make", [lambda: nn.Dropout(0.1), lambda: nn.Dropout(0.1, capturable=True), lambda: nn.AddNorm(8),
                                  lambda: nn.AddNorm(8, p=0.2, post_norm="rms", gate=True),
                                  lambda: nn.LinearCrossEntropy(8, 20)])
def test_layers_are_built_on_the_meta_device(make):
    with torch.device("meta"):
        m = make()
    assert all(t.is_meta for t in (*m.parameters(), *m.buffers()))


def test_draws_do_not_follow_the_default_device():
    torch.manual_seed(7)
    a = nn.Dropout(0.1)
    want = [a.seed, a.next_offset(), a.next_offset()]
    torch.manual_seed(7)
    with torch.device("meta"):
        b = nn.Dropout(0.1)
        assert [b.seed, b.next_offset(), b.next_offset()] == want


def test_layers_without_dropout_draw_nothing():
    torch.manual_seed(7)
    want = torch.rand(3)
    torch.manual_seed(7)
    nn.AddNorm(8), nn.Dropout(0.0)
    assert torch.equal(torch.rand(3), want)


def test_seeds():
    assert nn.Dropout(0.1, seed=5).seed == nn.Dropout(0.0, seed=5).seed == 5
    assert nn.Dropout(0.1).seed != nn.Dropout(0.1).seed
    assert nn.Dropout(0.0, capturable=True).seed != nn.Dropout(0.0, capturable=True).seed
    # made without dropout, given it later: the offsets still differ
    a, b = nn.Dropout(0.0), nn.Dropout(0.0)
    a.p = b.p = 0.5
    assert a.next_offset() != b.next_offset()
