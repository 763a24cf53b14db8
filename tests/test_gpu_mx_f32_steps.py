"""fp32 training steps on int8 checkpoints: with the exact sums' codes the gradients are those of the
definition but for fp32 sums."""
import numpy as np
import pytest
import torch

import oracle
from paper_2312_06881_amd.nn import DyadFF
from tests import mx_reference as ref
from tests.parity_util import TOL, to64
from workloads import layer_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("variant", ["IT", "OT", "DT"])
@pytest.mark.parametrize("shape", [(256, 512, 4, 129), (512, 1024, 8, 257), (1024, 2048, 2, 64), (96, 170, 5, 400), (770, 615, 5, 600)],
                         ids=lambda s: "x".join(map(str, s)))
def test_block_gradients(shape, variant):
    d, ffn, D, M = shape
    print("CASE mx8 f32 step", shape, variant, flush=True)
    A, B = layer_inputs(d, ffn, D, M, "f32", seed_offset=81), layer_inputs(ffn, d, D, M, "f32", seed_offset=82)
    m = DyadFF(d, ffn, D, variant, device="cuda", dtype=torch.float32, stash="mx8")
    with torch.no_grad():
        for mod, L in ((m.fc1, A), (m.fc2, B)):
            mod.w1.copy_(L.W1)
            mod.w2.copy_(L.W2)
            mod.bias.copy_(L.bias)
    x = A.X.cuda().requires_grad_(True)
    y = m(x)
    got = torch.autograd.grad(y, [x, m.fc1.w1, m.fc1.w2, m.fc1.bias, m.fc2.w1, m.fc2.w2, m.fc2.bias], B.dZ.cuda())
    w1a, w2a, ba = (A.f64(n) for n in ("W1", "W2", "bias"))
    w1b, w2b = B.f64("W1"), B.f64("W2")
    h = oracle.forward(variant, d, ffn, D, A.f64("X"), w1a, w2a, ba)
    hk, xk, dz = ref.values(torch.from_numpy(h).float().double().numpy(), "int8"), ref.values(A.f64("X"), "int8"), B.f64("dZ")
    dh = oracle.backward_dx(variant, ffn, d, D, dz, w1b, w2b, act_in=oracle.ACT_GELU, H_in=hk)
    want = (oracle.backward_dx(variant, d, ffn, D, dh, w1a, w2a), *oracle.backward_dw(variant, d, ffn, D, dh, xk),
            *oracle.backward_dw(variant, ffn, d, D, dz, oracle.gelu_array(hk)))
    # two fp32 sums in a row at most, each within a few 1e-6 of its largest value: the bar of one pass
    for g, r, name in zip(got, want, ("dx", "dW1a", "dW2a", "dba", "dW1b", "dW2b", "dbb")):
        e = np.abs(to64(g) - r).max() / np.abs(r).max()
        assert e <= TOL["f32"], (name, e)
