"""Passes over int8 checkpoints on a stream that no call has warmed up, captured into a graph: the
workspace that the library asks for is all they need."""
import numpy as np
import pytest
import torch

import oracle
from paper_2312_06881_amd import mx
from tests import mx_reference as ref
from tests.parity_util import assert_close
from workloads import layer_inputs

pytestmark = pytest.mark.gpu

SHAPES = [  # (n_in, n_out, n_dyad, tokens): split reductions, few tokens, columns that only buffered kernels take, copies
    (3072, 768, 4, 300),
    (1024, 1024, 8, 16),
    (768, 1536, 6, 200),
    (1024, 1024, 16, 200),
    (2048, 2048, 8, 2100),
    (770, 615, 5, 40),
]


@pytest.mark.parametrize("variant", ["IT", "OT", "DT"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_captured_on_a_cold_stream(shape, variant):
    n_in, n_out, D, M = shape
    print("CASE mx8 captured", shape, variant, flush=True)
    L = layer_inputs(n_in, n_out, D, M, "bf16", seed_offset=61)
    x, w1, w2, b, dz, h = (t.cuda() for t in (L.X, L.W1, L.W2, L.bias, L.dZ, L.H_in))

    def step():
        y, kept = mx.forward_gelu(x, w1, w2, b, variant)
        dx, a = mx.backward_dx_gelu(dz, w1, w2, mx.quantize(h), variant, want_act=True)
        return y, kept.dequantize(), dx, a

    eager = [t.clone() for t in step()]                     # on another stream than the capture's
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        out = step()
    rows = np.unique(np.linspace(0, M - 1, min(M, 60)).astype(int))
    at = torch.from_numpy(rows).cuda()
    hk = ref.values(L.f64("H_in"), "int8")
    first = (x.clone(), dz.clone(), h.clone())
    for shift in range(3):
        for t, t0 in zip((x, dz, h), first):
            t.copy_(t0.roll(shift, 0))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        src = (rows - shift) % M
        ry = oracle.forward(variant, n_in, n_out, D, L.f64("X")[src], L.f64("W1"), L.f64("W2"), L.f64("bias"),
                            act=oracle.ACT_GELU)
        rdx = oracle.backward_dx(variant, n_in, n_out, D, L.f64("dZ")[src], L.f64("W1"), L.f64("W2"),
                                 act_in=oracle.ACT_GELU, H_in=hk[src])
        assert_close(out[0][at], ry, "bf16", "Y")
        assert_close(out[2][at], rdx, "bf16", "dX")
        assert_close(out[3][at], oracle.gelu_array(hk[src]), "bf16", "GELU(H)")
        # sums in another order round the last bf16 bit of a value, and so its code, now and then
        same = (out[1] == eager[1].roll(shift, 0)).float().mean()
        assert same > 0.99, same
