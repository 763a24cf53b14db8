"""int8 blocks whose largest magnitude is 2^127 or more: the scale byte 254, whose codes reach
127 * 2^121, within fp32 and bf16."""
import numpy as np
import pytest
import torch

import oracle
from paper_2312_06881_amd import mx
from tests import mx_reference as ref
from tests.parity_util import assert_close
from workloads import layer_inputs

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def large(rows, cols, dtype, seed):
    """Blocks up to the type's largest value, of one sign, of both, and with zeros."""
    rng = np.random.default_rng(seed)
    top = float(torch.finfo(TORCH[dtype]).max)
    x = rng.uniform(-1, 1, (rows, cols)) * 2.0 ** 127 * rng.uniform(1, 1.99, (rows, 1))
    x[rng.random((rows, cols)) < 0.2] = 0.0
    x[::3] = np.abs(x[::3])
    x[1::3] = -np.abs(x[1::3])
    x[:, ::32] = 2.0 ** 127
    x[:, 1::32] = -top
    return torch.from_numpy(np.clip(x, -top, top)).float().to(TORCH[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 2), (66, 32), (9, 100), (257, 1001)], ids=lambda s: "x".join(map(str, s)))
def test_largest_blocks_read_back(shape, dtype):
    print("CASE mx largest blocks", shape, dtype, flush=True)
    x = large(*shape, dtype, 3)
    q = mx.quantize(x.cuda())
    codes, scales, values = ref.quantize(x.double().numpy(), "int8")
    assert (scales == 254).all()
    assert np.array_equal(q.scales.cpu().numpy(), scales) and np.array_equal(q.codes.cpu().numpy(), codes)
    for t in (torch.float32, torch.bfloat16):
        got = q.dequantize(t).cpu().double().numpy()
        assert np.isfinite(got).all() and np.array_equal(got, values)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("variant", ["IT", "OT", "DT"])
@pytest.mark.parametrize("shape", [(1024, 1024, 8, 16), (768, 768, 4, 300), (250, 154, 4, 65), (2048, 1024, 8, 2100),
                                   (1024, 4096, 4, 4100)], ids=lambda s: "x".join(map(str, s)))
def test_gradient_at_largest_blocks(shape, variant, dtype):
    """GELU' is 0 or 1 there and GELU(H) is 0 or H: in every pass that reads a checkpoint."""
    n_in, n_out, D, M = shape
    print("CASE mx dx at largest blocks", shape, variant, dtype, flush=True)
    L = layer_inputs(n_in, n_out, D, M, dtype, seed_offset=51)
    h = L.H_in.clone()
    rows = np.unique(np.linspace(0, M - 1, min(M, 60)).astype(int))
    h[rows, :64] = large(len(rows), 64, dtype, 4)
    kept = mx.quantize(h.cuda())
    dx, act = mx.backward_dx_gelu(L.dZ.cuda(), L.W1.cuda(), L.W2.cuda(), kept, variant, want_act=True)
    hk = ref.values(h.double().numpy()[rows], "int8")
    want = oracle.backward_dx(variant, n_in, n_out, D, L.f64("dZ")[rows], L.f64("W1"), L.f64("W2"),
                              act_in=oracle.ACT_GELU, H_in=hk)
    at = torch.from_numpy(rows).cuda()
    assert_close(dx[at], want, dtype, "dX")
    gelu = oracle.gelu_array(hk)
    assert_close(act[at][:, :64] / 2.0 ** 100, gelu[:, :64] / 2.0 ** 100, dtype, "GELU(H) of the largest blocks")
    assert_close(act[at][:, 64:], gelu[:, 64:], dtype, "GELU(H)")
