"""fp32 at n_dyad 1, where an output transpose leaves the columns consecutive."""
import pytest
import torch

import oracle
import paper_2312_06881_amd as dy
from tests.parity_util import assert_close
from workloads import layer_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("variant", ("IT", "OT", "DT"))
@pytest.mark.parametrize("shape", [(256, 256, 100), (128, 68, 7)], ids=lambda s: "x".join(map(str, s)))
def test_one_block(shape, variant):
    n_in, n_out, M = shape
    print("CASE f32 n_dyad 1", shape, variant, flush=True)
    L = layer_inputs(n_in, n_out, 1, M, "f32")
    x, w1, w2, b, dz, h = (t.to("cuda:0") for t in (L.X, L.W1, L.W2, L.bias, L.dZ, L.H_in))
    y, pre = dy.forward(x, w1, w2, b, variant=variant, act="gelu", stash_h=True)
    dx = dy.backward_dx(dz, w1, w2, variant, act_in="gelu", h_in=h)
    torch.cuda.synchronize()
    ry, rh = oracle.forward(variant, n_in, n_out, 1, L.f64("X"), L.f64("W1"), L.f64("W2"), L.f64("bias"),
                            act=oracle.ACT_GELU, want_h=True)
    rdx = oracle.backward_dx(variant, n_in, n_out, 1, L.f64("dZ"), L.f64("W1"), L.f64("W2"), act_in=oracle.ACT_GELU,
                             H_in=L.f64("H_in"))
    assert_close(y, ry, "f32", "Y")
    assert_close(pre, rh, "f32", "H")
    assert_close(dx, rdx, "f32", "dX")
