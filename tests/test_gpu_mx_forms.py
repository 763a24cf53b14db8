"""The fp4 product's kernels in both types, with and without GELU, at widths that end inside their
tiles, and with values that are not finite: every form that a batch or a few tokens choose."""
import math

import pytest
import torch

from paper_2312_06881_amd import mx
from paper_2312_06881_amd.nn import DyadFF, DyadLinear, MX4DyadFF
from tests import mx_reference as ref
from tests.parity_util import assert_close
from workloads import layer_inputs

pytestmark = pytest.mark.gpu

FORMS = [  # (n_in, n_out, n_dyad, tokens)
    (768, 1536, 4, 5000),      # large tiles; by residue, four fragments a wave in fp32
    (1024, 2048, 4, 4103),     # an odd batch
    (1152, 768, 4, 9001),
    (3072, 2048, 8, 1025),     # by residue, two fragments a wave in fp32
    (512, 4096, 8, 8200),
    (770, 2050, 4, 6000),      # padded: blocks of 193 and 513, rows no vector store fits
    (770, 2050, 4, 4100),
    (640, 2047, 1, 5003),      # one block, an odd width
    (768, 3080, 4, 8200),      # output transpose in LDS: blocks of 770
    (1200, 2400, 12, 8200),
    (640, 2560, 20, 3000),
    (1024, 2048, 32, 1100),
]


def case_id(s):
    return "x".join(map(str, s))


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("variant", ["IT", "OT", "DT"])
@pytest.mark.parametrize("shape", FORMS, ids=case_id)
def test_batches(shape, variant, dtype, act):
    """Rows that repeat 41 tokens: every place in the tiles gives the oracle's rows."""
    n_in, n_out, D, M = shape
    print("CASE mx4 form", shape, variant, dtype, act, flush=True)
    L = layer_inputs(n_in, n_out, D, 41, dtype, seed_offset=71)
    w = mx.quantize_weights(L.W1.cuda(), L.W2.cuda(), variant, n_in, n_out)
    x = L.X.cuda().repeat(M // 41 + 1, 1)[:M].contiguous()
    y = mx.forward(x, w, L.bias.cuda(), act=act)
    want = ref.mx4_forward(variant, n_in, n_out, D, L.f64("X"), L.f64("W1"), L.f64("W2"), L.f64("bias"), act)
    assert_close(y[:41], want, dtype, "Y")
    assert torch.equal(y, y[:41].repeat(M // 41 + 1, 1)[:M])


NON_FINITE = [  # few tokens quantised in place, small tiles, large tiles
    (256, 512, 4, 3),
    (1024, 2048, 4, 1),
    (1024, 2048, 4, 200),
    (1024, 2048, 4, 4103),
    (1024, 2048, 8, 4103),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("variant", ["IT", "OT", "DT"])
@pytest.mark.parametrize("shape", NON_FINITE, ids=case_id)
def test_non_finite_values(shape, variant, bad, dtype):
    """A token's value makes NaN of the outputs that read its 32 in either component, a weight's of
    its output for every token; the others keep their bits."""
    n_in, n_out, D, M = shape
    print("CASE mx4 non-finite", shape, variant, bad, dtype, flush=True)
    bi, bo = n_in // D, n_out // D
    L = layer_inputs(n_in, n_out, D, M, dtype, seed_offset=72)
    x, w1, w2 = L.X.cuda(), L.W1.cuda(), L.W2.cuda()
    y = mx.forward(x, mx.quantize_weights(w1, w2, variant), L.bias.cuda())
    assert y.isfinite().all()
    m, c, (g, j, k) = M - 1, bi + 5, (D - 1, bo - 3, 7)
    bad_x, bad_w = x.clone(), w1.clone()
    bad_x[m, c] = bad
    bad_w[g, j, k] = bad
    f = torch.arange(n_out, device=x.device)
    reads = f // bo == 1                                               # component 1: the value's block
    block2 = c % D if variant in ("IT", "DT") else 1                   # component 2: its residue or block
    reads |= (f % D if variant in ("OT", "DT") else f // bo) == block2
    want = torch.zeros(M, n_out, dtype=torch.bool, device=x.device)
    want[m] = reads
    z = mx.forward(bad_x, mx.quantize_weights(w1, w2, variant), L.bias.cuda())
    assert torch.equal(z.isnan(), want) and torch.equal(z[~want], y[~want])
    want = torch.zeros_like(want)
    want[:, g * bo + j] = True
    z = mx.forward(x, mx.quantize_weights(bad_w, w2, variant), L.bias.cuda())
    assert torch.equal(z.isnan(), want) and torch.equal(z[~want], y[~want])


def test_modules_behind_a_trainable_layer():
    """Inference where a gradient is recorded gives the same outputs, and a backward pass is refused."""
    torch.manual_seed(5)
    served = MX4DyadFF(DyadFF(256, 1024, 4, ("IT", "DT"), device="cuda"))
    front = DyadLinear(256, 256, 4, "OT", device="cuda")
    x = torch.randn(3, 70, 256, device="cuda").bfloat16()
    h = front(x)
    y = served(h)
    assert y.requires_grad
    with torch.no_grad():
        assert torch.equal(served(front(x)), y)
    with pytest.raises(NotImplementedError, match="gradient"):
        (h + y).float().sum().backward()
    assert front.w1.grad is None
