"""State dicts of the fp4 modules: packed weights of another layer are not taken for this one's."""
import copy

import pytest
import torch

import paper_2312_06881_amd as dy
from paper_2312_06881_amd import mx
from paper_2312_06881_amd.nn import DyadFF, DyadLinear, MX4DyadFF, MX4DyadLinear


@pytest.fixture(autouse=True)
def packed_on_the_cpu(monkeypatch):
    def quantize_weights(w1, w2, variant="IT", n_in=None, n_out=None):
        need = dy.dyad_mx4_weight_bytes(dy.VARIANTS[variant], n_in, n_out, w1.shape[0])
        return mx.MX4Weights(torch.randint(0, 256, (need,), dtype=torch.uint8), variant, n_in, n_out, w1.shape[0])

    monkeypatch.setattr(mx, "quantize_weights", quantize_weights)


def served(n_in=64, n_out=256, D=4, variant="IT", bias=True):
    return MX4DyadLinear(DyadLinear(n_in, n_out, D, variant, bias=bias))


@pytest.mark.parametrize("other", [dict(variant="OT"), dict(variant="DT"), dict(D=2), dict(n_in=60), dict(n_in=100), dict(n_out=250)],
                         ids=str)
@pytest.mark.parametrize("strict", [True, False])
def test_another_layers_weights_are_refused(other, strict):
    m, state = served(bias=False), served(bias=False, **other).state_dict()
    kept = m.packed.clone()
    with pytest.raises(RuntimeError, match="packed"):
        m.load_state_dict(state, strict=strict)
    assert torch.equal(m.packed, kept)


def test_another_layout_is_refused():
    m = served()
    state = copy.deepcopy(m.state_dict())
    state["layout"][0] += 1
    with pytest.raises(RuntimeError, match="packed"):
        m.load_state_dict(state)


@pytest.mark.parametrize("assign", [False, True])
def test_the_same_layers_weights_load(assign):
    a, b = served(variant="DT"), served(variant="DT")
    assert not torch.equal(a.packed, b.packed)
    b.load_state_dict(a.state_dict(), assign=assign)
    assert torch.equal(a.packed, b.packed) and torch.equal(a.bias, b.bias)


def test_a_block_and_states_without_the_layout():
    a, b = (MX4DyadFF(DyadFF(64, 256, 4, ("IT", "OT"))) for _ in range(2))
    state = a.state_dict()
    before = {k: v for k, v in state.items() if not k.endswith("layout")}
    assert set(before) == {"fc1.packed", "fc1.bias", "fc2.packed", "fc2.bias"}
    b.load_state_dict(before)
    assert torch.equal(a.fc2.packed, b.fc2.packed)
    with pytest.raises(RuntimeError, match="packed"):
        MX4DyadFF(DyadFF(64, 256, 4, ("IT", "DT"))).load_state_dict(state)
    # no part of the module itself: what it holds is its weights and bias
    assert [n for n, _ in a.named_buffers()] == ["fc1.packed", "fc1.bias", "fc2.packed", "fc2.bias"]
