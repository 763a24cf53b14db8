"""fp32 passes whose operands lie n_dyad apart: the widest tiles keep them, and the weight gradient's
128 x 64 and 64 x 128 among those."""
import numpy as np
import pytest

import oracle
import paper_2312_06881_amd as dy
from tests.parity_util import assert_close, to64
from workloads import layer_inputs

pytestmark = pytest.mark.gpu

DW = [  # (n_in, n_out, n_dyad, tokens): blocks of 32 x 128, 128 x 32, 128 x 128 and, with the last ones short, 24 x 96
    (1024, 4096, 32, 2048),
    (4096, 1024, 32, 2000),
    (4096, 4096, 32, 1536),
    (768, 3072, 32, 1550),
]


@pytest.mark.parametrize("variant", ["IT", "OT", "DT"])
@pytest.mark.parametrize("shape", DW, ids=lambda s: "x".join(map(str, s)))
def test_weight_gradient(shape, variant):
    n_in, n_out, D, M = shape
    print("CASE f32 gathers dw", shape, variant, flush=True)
    L = layer_inputs(n_in, n_out, D, M, "f32", seed_offset=91)
    dw1, dw2, db = dy.backward_dw(L.dZ.cuda(), L.X.cuda(), D, variant)
    rng = np.random.default_rng(6)
    comp = rng.integers(1, 3, 600)
    g, j, k = (rng.integers(0, n, 600) for n in (D, n_out // D, n_in // D))
    want = oracle.backward_dw_entries(variant, n_in, n_out, D, L.f64("dZ"), L.f64("X"), comp, g, j, k)
    assert_close(np.where(comp == 1, to64(dw1)[g, j, k], to64(dw2)[g, j, k]), want, "f32", "dW entries")
    assert_close(db, L.f64("dZ").sum(0), "f32", "db")


@pytest.mark.parametrize("shape", [(512, 2048, 8, 2048), (4096, 1024, 16, 1024), (1024, 4096, 32, 1024), (768, 3072, 32, 1500)],
                         ids=lambda s: "x".join(map(str, s)))
def test_forward_and_input_gradient(shape):
    n_in, n_out, D, M = shape
    print("CASE f32 gathers", shape, flush=True)
    L = layer_inputs(n_in, n_out, D, M, "f32", seed_offset=92)
    rows = np.unique(np.linspace(0, M - 1, 100).astype(int))
    y = dy.forward(L.X.cuda(), L.W1.cuda(), L.W2.cuda(), L.bias.cuda(), "IT")
    want = oracle.forward("IT", n_in, n_out, D, L.f64("X")[rows], L.f64("W1"), L.f64("W2"), L.f64("bias"))
    assert_close(to64(y)[rows], want, "f32", "Y")
    dx = dy.backward_dx(L.dZ.cuda(), L.W1.cuda(), L.W2.cuda(), "OT")
    want = oracle.backward_dx("OT", n_in, n_out, D, L.f64("dZ")[rows], L.f64("W1"), L.f64("W2"))
    assert_close(to64(dx)[rows], want, "f32", "dX")
