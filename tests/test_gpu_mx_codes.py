"""The fp32 forward pass that keeps its pre-activation: the codes are those of the exact sums."""
import numpy as np
import pytest
import torch

import oracle
from paper_2312_06881_amd import mx
from tests import mx_reference as ref
from workloads import layer_inputs

pytestmark = pytest.mark.gpu

SHAPES = [  # (n_in, n_out, n_dyad, tokens): tiles of every size, and blocks that no tile takes
    (768, 3072, 4, 700),
    (2048, 1024, 8, 1030),
    (1024, 1024, 16, 300),
    (256, 256, 1, 100),
    (64, 256, 2, 1),
    (250, 154, 4, 65),        # padded widths
    (770, 615, 5, 600),
    (768, 3072, 5, 300),      # blocks of 154 and 615
    (90, 150, 3, 257),        # blocks of 30 and 50
    (7, 33, 2, 40),
    (40, 8, 16, 129),         # more blocks than columns
]


@pytest.mark.parametrize("variant", ["IT", "OT", "DT"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_codes_are_those_of_the_exact_sums(shape, variant):
    """Every code and scale byte is that of the oracle's 64-bit pre-activation rounded once to
    fp32: a sum in 64 bits is near enough to it for no value here to lie between the two."""
    n_in, n_out, D, M = shape
    print("CASE mx codes", shape, variant, flush=True)
    L = layer_inputs(n_in, n_out, D, M, "f32", seed_offset=41)
    y, kept = mx.forward_gelu(L.X.cuda(), L.W1.cuda(), L.W2.cuda(), L.bias.cuda(), variant)
    rows = np.unique(np.linspace(0, M - 1, min(M, 300)).astype(int))
    h = oracle.forward(variant, n_in, n_out, D, L.f64("X")[rows], L.f64("W1"), L.f64("W2"), L.f64("bias"))
    codes, scales, _ = ref.quantize(torch.from_numpy(h).float().double().numpy(), "int8")
    assert np.array_equal(kept.scales.cpu().numpy()[rows], scales)
    assert np.array_equal(kept.codes.cpu().numpy()[rows], codes)
