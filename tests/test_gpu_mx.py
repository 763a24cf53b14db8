"""Microscaled operators on the GPU against their definition in 64 bits: quantised
values exactly, the fp4 product and the passes over int8 checkpoints within what their
arithmetic allows (parity_util: one rounding of an fp32 sum)."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2312_06881_amd as dy
from paper_2312_06881_amd import mx
from paper_2312_06881_amd.nn import DyadFF, DyadLinear, MX4DyadFF, MX4DyadLinear
from tests import mx_reference as ref
from tests.parity_util import assert_close, to64
from workloads import draw, layer_inputs

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
VARIANTS = ("IT", "OT", "DT")
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def banner(*what):
    print("CASE mx", *what, flush=True)


def exact64(t):
    return t.detach().cpu().to(torch.float64).numpy()


# ---- quantisation ------------------------------------------------------------------

def sample(rows, cols, dtype, seed):
    """Normal values at magnitudes from 2^-140 to 2^120, rows of zeros, and values on and
    next to the midpoints between elements."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols))
    x *= np.exp2(rng.integers(-140, 120, (rows, 1)) * (rng.random((rows, 1)) < 0.5))
    x[rng.random(rows) < 0.1] = 0.0
    ties = rng.integers(-48, 49, (rows, cols)) / 8.0 * np.exp2(rng.integers(-3, 3, (rows, 1)))
    x = np.where(rng.random((rows, 1)) < 0.3, ties, x)
    return torch.from_numpy(x).to(torch.float32).to(TORCH[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp4"])
@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (257, 31), (64, 32), (65, 33), (129, 40), (33, 100), (17, 1024),
                                   (1000, 770), (5, 4099)], ids=lambda s: "x".join(map(str, s)))
def test_quantize_is_exact(shape, fmt, dtype):
    rows, cols = shape
    banner("quantize", shape, fmt, dtype)
    x = sample(rows, cols, dtype, 7 * rows + cols)
    q = mx.quantize(x.to(DEV), fmt)
    back = q.dequantize()
    back32 = q.dequantize(torch.float32)
    torch.cuda.synchronize()
    codes, scales, values = ref.quantize(exact64(x), fmt)
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    got = q.codes.cpu().numpy().astype(np.int64)
    if fmt == "fp4":
        nib = np.stack([got & 15, got >> 4], -1).reshape(rows, -1)
        if cols % 2:
            assert not nib[:, cols].any()
        nib = nib[:, :cols]
        got = np.where(nib & 8, -(nib & 7), nib & 7)
    assert np.array_equal(got, codes)
    assert back.dtype == x.dtype and back.shape == x.shape
    assert np.array_equal(exact64(back32), values)
    assert np.array_equal(exact64(back), exact64(torch.from_numpy(values).to(torch.float32).to(TORCH[dtype])))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "fp4"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_non_finite_blocks_read_back_as_nan(bad, fmt, dtype):
    x = torch.ones(4, 100, dtype=TORCH[dtype])
    x[1, 40] = bad
    x[2, 99] = bad
    got = mx.quantize(x.to(DEV), fmt).dequantize().cpu()
    want = torch.zeros(4, 100, dtype=torch.bool)
    want[1, 32:64] = True
    want[2, 96:] = True
    assert torch.equal(got.isnan(), want)
    assert torch.equal(got[~want], x[~want])


def test_quantize_empty_and_leading_dimensions():
    q = mx.quantize(torch.zeros(0, 33, device=DEV))
    assert q.dequantize().shape == (0, 33)
    x = torch.randn(2, 3, 40, device=DEV).bfloat16()
    a, b = mx.quantize(x), mx.quantize(x.view(6, 40))
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    assert a.dequantize().shape == x.shape
    assert a.nbytes == 6 * 40 + 6 * 2


def test_offsets_past_32_bits():
    """2^31 codes and more: the last rows land where they belong."""
    rows, cols = 66000, 32800
    banner("large", rows, cols)
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    tail = torch.randn(3, cols, device=DEV).bfloat16()
    x[-3:] = tail
    q = mx.quantize(x)
    small = mx.quantize(tail)
    assert torch.equal(q.codes[-3:], small.codes) and torch.equal(q.scales[-3:], small.scales)
    del x
    assert torch.equal(q.dequantize()[-3:], small.dequantize())


# ---- the fp4 product ---------------------------------------------------------------

PRODUCT = [  # (n_in, n_out, n_dyad, tokens)
    (768, 768, 4, 1),
    (1024, 192, 4, 7),        # few tokens: a block that ends inside a step
    (160, 64, 4, 3),          # and inside a block of 32
    (256, 512, 4, 16),
    (1024, 512, 2, 16),
    (512, 256, 2, 17),
    (64, 64, 1, 33),          # blocks shorter than one matrix step
    (250, 154, 4, 65),        # widths n_dyad does not divide
    (770, 615, 5, 130),
    (100, 300, 7, 3),         # blocks of 15 and 43
    (96, 93, 3, 20),
    (2048, 1024, 16, 66),
    (512, 512, 16, 129),
    (1200, 720, 12, 31),
    (640, 1280, 20, 40),
    (8, 8, 16, 5),            # more blocks than columns
    (4096, 64, 8, 200),
    (1100, 2112, 6, 257),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("shape", PRODUCT, ids=lambda s: "x".join(map(str, s)))
def test_mx4_forward(shape, variant, dtype):
    n_in, n_out, D, M = shape
    act = "gelu" if (n_in + M) % 2 else "none"
    banner("product", shape, variant, dtype, act)
    L = layer_inputs(n_in, n_out, D, M, dtype, seed_offset=11)
    w = mx.quantize_weights(L.W1.to(DEV), L.W2.to(DEV), variant, n_in, n_out)
    y = mx.forward(L.X.to(DEV), w, L.bias.to(DEV), act=act)
    torch.cuda.synchronize()
    want = ref.mx4_forward(variant, n_in, n_out, D, L.f64("X"), L.f64("W1"), L.f64("W2"), L.f64("bias"), act)
    assert_close(y, want, dtype, "Y")


MANY = [  # (n_in, n_out, n_dyad, tokens): every form of the large tiles, last panels of a few tokens
    (768, 1536, 4, 5000),
    (1024, 2048, 4, 4103),    # blocks of two steps
    (4096, 4096, 4, 6000),
    (512, 4096, 8, 8200),     # one step: an odd number in each component
    (3072, 2048, 8, 1025),    # three
    (2048, 4096, 16, 3333),
    (2048, 8192, 16, 2049),
    (1152, 768, 4, 9001),
    (1536, 1536, 3, 4097),
]


@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("shape", MANY, ids=lambda s: "x".join(map(str, s)))
def test_mx4_forward_many_tokens(shape, variant):
    """Rows that repeat 37 tokens: every place in the large tiles gives the oracle's rows."""
    n_in, n_out, D, M = shape
    banner("product, many tokens", shape, variant)
    L = layer_inputs(n_in, n_out, D, 37, "bf16", seed_offset=12)
    w = mx.quantize_weights(L.W1.to(DEV), L.W2.to(DEV), variant)
    x = L.X.to(DEV).repeat(M // 37 + 1, 1)[:M].contiguous()
    y = mx.forward(x, w, L.bias.to(DEV))
    want = ref.mx4_forward(variant, n_in, n_out, D, L.f64("X"), L.f64("W1"), L.f64("W2"), L.f64("bias"), "none")
    assert_close(y[:37], want, "bf16", "Y")
    assert torch.equal(y, y[:37].repeat(M // 37 + 1, 1)[:M])


def test_mx4_no_bias_no_tokens_and_own_workspace():
    L = layer_inputs(256, 512, 4, 39, "bf16")
    w = mx.quantize_weights(L.W1.to(DEV), L.W2.to(DEV), "DT")
    x = L.X.to(DEV)
    assert mx.forward(x[:0], w).shape == (0, 512)
    y = mx.forward(x, w)
    ws = torch.full((dy.dyad_mx4_workspace_bytes(dy.DT, 256, 512, 4, 39),), 255, dtype=torch.uint8, device=DEV)
    assert torch.equal(mx.forward(x, w, workspace=ws), y)
    with pytest.raises(dy.DyadError) as e:
        mx.forward(x, w, workspace=ws[:-1])
    assert e.value.status == -5


@pytest.mark.parametrize("variant", VARIANTS)
def test_mx4_non_finite_input(variant):
    """A token's infinity reaches the outputs that read its block, and no other token."""
    L = layer_inputs(256, 256, 4, 40, "bf16")
    w = mx.quantize_weights(L.W1.to(DEV), L.W2.to(DEV), variant)
    x = L.X.to(DEV)
    y = mx.forward(x, w)
    x[7, 70] = math.inf
    z = mx.forward(x, w)
    others = torch.arange(40, device=DEV) != 7
    assert torch.equal(z[others], y[others])
    row = z[7].isnan()
    assert row[64:128].all()                                  # component 1's block 1
    if variant == "IT":                                       # and component 2's residue 70 % 4
        assert row[128:192].all() and not row[:64].any() and not row[192:].any()


def test_mx4_modules():
    torch.manual_seed(3)
    ff = DyadFF(256, 1024, 4, ("IT", "DT"), device=DEV)
    x = torch.randn(2, 19, 256, device=DEV).bfloat16()
    served = MX4DyadFF(ff)
    y = served(x)
    assert y.shape == x.shape and not y.requires_grad
    a = ref.mx4_forward("IT", 256, 1024, 4, exact64(x).reshape(38, 256), exact64(ff.fc1.w1), exact64(ff.fc1.w2),
                        exact64(ff.fc1.bias), "gelu")
    assert_close(served.fc1(x).reshape(38, 1024), a, "bf16", "fc1")
    z = served.fc1(x).reshape(38, 1024)
    b = ref.mx4_forward("DT", 1024, 256, 4, exact64(z), exact64(ff.fc2.w1), exact64(ff.fc2.w2), exact64(ff.fc2.bias),
                        "none")
    assert_close(y.reshape(38, 256), b, "bf16", "Y")
    other = MX4DyadLinear(DyadLinear(256, 1024, 4, "IT", device=DEV), "gelu")
    other.load_state_dict(served.fc1.state_dict())
    assert torch.equal(other(x), served.fc1(x))


# ---- int8 checkpoints --------------------------------------------------------------

PASSES = [  # (n_in, n_out, n_dyad, tokens): small batches, tiles, narrow and padded blocks, large batches
    (768, 3072, 4, 1),
    (1024, 1024, 8, 16),
    (768, 3072, 4, 700),
    (3072, 768, 4, 515),
    (2048, 1024, 8, 1030),
    (1024, 1024, 16, 2100),
    (256, 256, 1, 100),
    (250, 154, 4, 65),
    (770, 615, 5, 600),
    (768, 1536, 6, 2050),
    (512, 384, 2, 33),
    (1024, 4096, 4, 4100),
]


def gelu64(x):
    return oracle.gelu_array(x)


def case_id(s):
    return "x".join(map(str, s))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("shape", PASSES, ids=case_id)
def test_forward_keeps_the_quantised_preactivation(shape, variant, dtype):
    """The checkpoint is the quantised H of dyad_forward: bit for bit where that pass sums in the same
    order, and else within a step wherever H itself is within its own rounding of the oracle's."""
    n_in, n_out, D, M = shape
    banner("forward", shape, variant, dtype)
    L = layer_inputs(n_in, n_out, D, M, dtype, seed_offset=21)
    t = [L.X.to(DEV), L.W1.to(DEV), L.W2.to(DEV), L.bias.to(DEV)]
    y, kept = mx.forward_gelu(*t, variant=variant)
    torch.cuda.synchronize()
    rows = np.unique(np.linspace(0, M - 1, min(M, 200)).astype(int))
    ry, rh = oracle.forward(variant, n_in, n_out, D, L.f64("X")[rows], L.f64("W1"), L.f64("W2"), L.f64("bias"),
                            act=oracle.ACT_GELU, want_h=True)
    at = torch.from_numpy(rows).to(DEV)
    assert_close(y[at], ry, dtype, "Y")
    # |kept - h| <= half a step of the block, and 2^-8 of the value (its rounding to bf16) with the fp32 sum's error;
    # a largest value that rounds up to the next power of two doubles the step
    got = exact64(kept.dequantize(torch.float32))[rows]
    # codes saturate at 127 / 64, half a step more below the next power of two
    step = np.exp2(np.repeat(kept.scales.cpu().numpy().astype(np.float64)[rows] - 133, 32, axis=1)[:, :n_out])
    err = 2.0 ** -8 * np.abs(rh) + 2.0 ** -10 * np.abs(rh).max() if dtype == "bf16" else 1e-6 * np.abs(rh) + 2e-6 * np.abs(rh).max()
    assert (np.abs(got - rh) <= np.where(np.abs(got) >= 127 * step, 1.0, 0.5) * step + err).all()
    h = dy.forward(*t, variant=variant, act="gelu", stash_h=True)[1]
    q = mx.quantize(h)
    same = (kept.codes == q.codes).float().mean()
    assert same > 0.99, same


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("shape", PASSES, ids=case_id)
def test_backward_dx(shape, variant, dtype):
    n_in, n_out, D, M = shape
    banner("dx", shape, variant, dtype)
    L = layer_inputs(n_in, n_out, D, M, dtype, seed_offset=22)
    kept = mx.quantize(L.H_in.to(DEV))
    args = (L.dZ.to(DEV), L.W1.to(DEV), L.W2.to(DEV), kept, variant)
    dx = mx.backward_dx_gelu(*args)
    again, act = mx.backward_dx_gelu(*args, want_act=True)
    torch.cuda.synchronize()
    assert torch.equal(dx, again)
    rows = np.unique(np.linspace(0, M - 1, min(M, 200)).astype(int))
    hk = ref.values(L.f64("H_in")[rows], "int8")
    want = oracle.backward_dx(variant, n_in, n_out, D, L.f64("dZ")[rows], L.f64("W1"), L.f64("W2"),
                              act_in=oracle.ACT_GELU, H_in=hk)
    assert_close(dx[torch.from_numpy(rows).to(DEV)], want, dtype, "dX")
    assert_close(act[torch.from_numpy(rows).to(DEV)], gelu64(hk), dtype, "GELU(H)")


@pytest.mark.parametrize("act_in", ["none", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("shape", PASSES, ids=case_id)
def test_backward_dw(shape, variant, dtype, act_in):
    n_in, n_out, D, M = shape
    banner("dw", shape, variant, dtype, act_in)
    L = layer_inputs(n_in, n_out, D, M, dtype, seed_offset=23)
    kept = mx.quantize(L.X.to(DEV))
    dw1, dw2, db = mx.backward_dw(L.dZ.to(DEV), kept, D, variant, act_in=act_in)
    again = mx.backward_dw(L.dZ.to(DEV), kept, D, variant, want_db=False, act_in=act_in)
    torch.cuda.synchronize()
    assert torch.equal(dw1, again[0]) and torch.equal(dw2, again[1]) and again[2] is None
    x = ref.values(L.f64("X"), "int8")
    if act_in == "gelu":
        # the layer's input, rounded to its type as the activation between two layers is
        x = exact64(torch.from_numpy(gelu64(x)).to(TORCH[dtype]))
    dz = L.f64("dZ")
    if M * n_in * n_out > 2 ** 28:                            # the oracle's loops: a part of the entries
        rng = np.random.default_rng(5)
        comp = rng.integers(1, 3, 400)
        g, j, k = (rng.integers(0, n, 400) for n in (D, -(-n_out // D), -(-n_in // D)))
        want = oracle.backward_dw_entries(variant, n_in, n_out, D, dz, x, comp, g, j, k)
        got = np.where(comp == 1, to64(dw1)[g, j, k], to64(dw2)[g, j, k])
        assert_close(got, want, dtype, "dW entries")
        assert_close(db, dz.sum(0), dtype, "db")
        return
    r1, r2, rb = oracle.backward_dw(variant, n_in, n_out, D, dz, x)
    assert_close(dw1, r1, dtype, "dW1")
    assert_close(dw2, r2, dtype, "dW2")
    assert_close(db, rb, dtype, "db")


def test_empty_batch():
    w = torch.randn(4, 64, 32, device=DEV).bfloat16()
    y, kept = mx.forward_gelu(torch.zeros(0, 128, device=DEV).bfloat16(), w, w)
    assert y.shape == (0, 256) and kept.codes.shape == (0, 256)
    assert mx.backward_dx_gelu(torch.zeros(0, 256, device=DEV).bfloat16(), w, w,
                               mx.quantize(torch.zeros(0, 128, device=DEV).bfloat16())).shape == (0, 128)
    dw1, dw2, db = mx.backward_dw(torch.zeros(0, 256, device=DEV).bfloat16(),
                                  mx.quantize(torch.zeros(0, 128, device=DEV).bfloat16()), 4)
    assert not dw1.any() and not dw2.any() and not db.any()


def test_non_finite_checkpoint_reaches_the_gradients():
    """A NaN block of the checkpoint gives NaN where it is read: those columns of dX and of dW."""
    L = layer_inputs(256, 256, 4, 70, "bf16")
    h = L.X.to(DEV)
    h[5, 33] = math.nan
    kept = mx.quantize(h)
    dx = mx.backward_dx_gelu(L.dZ.to(DEV), L.W1.to(DEV), L.W2.to(DEV), kept, "IT")
    want = torch.zeros(70, 256, dtype=torch.bool, device=DEV)
    want[5, 32:64] = True
    assert torch.equal(dx.isnan(), want)
    dw1, _, db = mx.backward_dw(L.dZ.to(DEV), kept, 4, "OT", act_in="gelu")
    assert dw1[0, :, 32:64].isnan().all() and not dw1[0, :, :32].isnan().any() and not dw1[1:].isnan().any()
    assert not db.isnan().any()


# ---- the modules -------------------------------------------------------------------

def ff_reference(variant, D, x, dz, p, dtype):
    """(y, dx, dW1a, dW2a, dba, dW1b, dW2b, dbb) of a block in 64 bits, from the checkpoints' definition."""
    (w1a, w2a, ba), (w1b, w2b, bb) = p
    d, ffn = x.shape[1], ba.shape[0]
    a, h = oracle.forward(variant, d, ffn, D, x, w1a, w2a, ba, act=oracle.ACT_GELU, want_h=True)
    y = oracle.forward(variant, ffn, d, D, a, w1b, w2b, bb)
    hk = ref.values(exact64(torch.from_numpy(h).to(TORCH[dtype])), "int8")
    xk = ref.values(x, "int8")
    dh = oracle.backward_dx(variant, ffn, d, D, dz, w1b, w2b, act_in=oracle.ACT_GELU, H_in=hk)
    dx = oracle.backward_dx(variant, d, ffn, D, dh, w1a, w2a)
    return (y, dx, *oracle.backward_dw(variant, d, ffn, D, dh, xk),
            *oracle.backward_dw(variant, ffn, d, D, dz, oracle.gelu_array(hk)))


def ff_setup(variant, D, d, ffn, M, dtype, stash="mx8"):
    A, B = layer_inputs(d, ffn, D, M, dtype, seed_offset=31), layer_inputs(ffn, d, D, M, dtype, seed_offset=32)
    m = DyadFF(d, ffn, D, variant, device=DEV, dtype=TORCH[dtype], stash=stash)
    with torch.no_grad():
        for mod, L in ((m.fc1, A), (m.fc2, B)):
            mod.w1.copy_(L.W1)
            mod.w2.copy_(L.W2)
            mod.bias.copy_(L.bias)
    params = [(L.f64("W1"), L.f64("W2"), L.f64("bias")) for L in (A, B)]
    return m, A.X, B.dZ, A.f64("X"), B.f64("dZ"), params


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("shape", [(256, 512, 4, 129), (96, 170, 5, 40)], ids=case_id)
def test_ff_step(shape, variant, dtype):
    d, ffn, D, M = shape
    banner("ff", shape, variant, dtype)
    m, x, dz, x64, dz64, params = ff_setup(variant, D, d, ffn, M, dtype)
    x = x.to(DEV).requires_grad_(True)
    y = m(x)
    got = (y, *torch.autograd.grad(y, [x, m.fc1.w1, m.fc1.w2, m.fc1.bias, m.fc2.w1, m.fc2.w2, m.fc2.bias], dz.to(DEV)))
    want = ff_reference(variant, D, x64, dz64, params, dtype)
    # bf16: each result is a sum over an operand rounded to bf16 (relative 2^-9 each, independent) and is
    # rounded itself: max-norm 2e-2 as elsewhere.  fp32: a pre-activation whose fp32 sum falls on the other
    # side of a rounding boundary moves one checkpointed value by a step, 2^-6 of its block's largest
    for g, r, name in zip(got, want, ("y", "dx", "dW1a", "dW2a", "dba", "dW1b", "dW2b", "dbb")):
        e = np.abs(to64(g) - r).max() / np.abs(r).max()
        assert e <= (2e-2 if dtype == "bf16" else 2e-3), (name, e)


def test_gradient_against_differences():
    """fp32 gradients against central differences of the block linearised at its checkpoints:
    x enters the loss through GELU at kept_h + (h(x') - h(x)), the weights of fc1 through the kept x."""
    variant, D, d, ffn, M = "DT", 4, 64, 128, 33
    m, x, dz, x64, dz64, params = ff_setup(variant, D, d, ffn, M, "f32")
    x = x.to(DEV).requires_grad_(True)
    leaves = [x, m.fc1.w1, m.fc1.bias, m.fc2.w2]
    grads = [exact64(g) for g in torch.autograd.grad(m(x), leaves, dz.to(DEV))]
    (w1a, w2a, ba), (w1b, w2b, bb) = params
    h0 = oracle.forward(variant, d, ffn, D, x64, w1a, w2a, ba)
    hk, xk = ref.values(exact64(torch.from_numpy(h0).float()), "int8"), ref.values(x64, "int8")

    def loss(dx=0.0, dw1=0.0, dbias=0.0, dw2b=0.0):
        # the pre-activation's change, through x as it was and the weights at the kept x
        dh = oracle.forward(variant, d, ffn, D, x64 + dx, w1a, w2a, ba) - h0
        dh = dh + oracle.forward(variant, d, ffn, D, xk, w1a + dw1, w2a, ba + dbias)
        dh = dh - oracle.forward(variant, d, ffn, D, xk, w1a, w2a, ba)
        return (oracle.forward(variant, ffn, d, D, oracle.gelu_array(hk + dh), w1b, w2b + dw2b, bb) * dz64).sum()

    rng = np.random.default_rng(9)
    for name, g in zip(("dx", "dw1", "dbias", "dw2b"), grads):
        v = rng.standard_normal(g.shape)
        eps = 1e-5
        num = (loss(**{name: eps * v}) - loss(**{name: -eps * v})) / (2 * eps)
        # differences: O(eps^2); fp32 gradients and a rounding flip of a kept value: 2e-3 as above
        assert abs(num - (g * v).sum()) <= 2e-3 * np.sqrt((g ** 2).sum() * (v ** 2).sum()), name


def test_linear_step_strides_and_broadcast_gradients():
    torch.manual_seed(1)
    m = DyadLinear(256, 384, 4, "OT", device=DEV, stash="mx8")
    base = torch.randn(256, 50, device=DEV).bfloat16()
    x = base.t().unsqueeze(0).expand(2, 50, 256).requires_grad_(True)     # not contiguous, shared over the batch
    y = m(x)
    grads = torch.autograd.grad(y.float().sum(), [x, m.w1, m.w2, m.bias])  # an expanded upstream gradient
    flat = x.detach().reshape(100, 256).contiguous()
    ones = torch.ones(100, 384, device=DEV).bfloat16()
    want = mx.backward_dw(ones, mx.quantize(flat), 4, "OT")
    assert torch.equal(y.reshape(100, 384), dy.forward(flat, m.w1.detach(), m.w2.detach(), m.bias.detach(), "OT"))
    assert torch.equal(grads[0].reshape(100, 256), dy.backward_dx(ones, m.w1.detach(), m.w2.detach(), "OT"))
    for a, b in zip(grads[1:], want):
        assert torch.equal(a, b)


def test_only_what_is_read_is_kept():
    m = DyadFF(256, 1024, 4, "IT", device=DEV, stash="mx8")
    plain = DyadFF(256, 1024, 4, "IT", device=DEV)
    plain.load_state_dict(m.state_dict())
    x = torch.randn(130, 256, device=DEV).bfloat16()

    def saved(mod, inp):
        n = []
        with torch.autograd.graph.saved_tensors_hooks(lambda t: (n.append(t.nbytes), t)[1], lambda t: t):
            y = mod(inp)
        return y, sum(n) - sum(p.nbytes for p in mod.parameters() if p.dim() == 3)

    y, kept = saved(m, x)
    z, full = saved(plain, x)
    assert torch.equal(y, z)
    assert kept == 130 * (256 + 8 + 1024 + 32)                # codes and scales of x and h
    assert full >= 2 * 130 * (256 + 2 * 1024)
    for p in (m.fc1.w1, m.fc1.w2, m.fc1.bias):
        p.requires_grad_(False)
    y, kept = saved(m, x)
    assert kept == 130 * (1024 + 32)
    y.sum().backward()
    assert m.fc2.w1.grad is not None and m.fc1.w1.grad is None
    with torch.no_grad():
        assert torch.equal(m(x), y.detach())


def test_other_stream_and_graph_replays():
    """Each call works on torch's current stream, and replays of a captured graph (several, with eager
    work between them) give the eager results."""
    torch.manual_seed(2)
    m = DyadFF(256, 512, 4, "DT", device=DEV, stash="mx8")
    served = MX4DyadFF(m)
    x = torch.randn(300, 256, device=DEV).bfloat16()
    dz = torch.randn(300, 256, device=DEV).bfloat16()

    def step():
        xi = x.detach().requires_grad_(True)
        y = m(xi)
        return (y.detach(), served(x), mx.quantize(x, "fp4").dequantize(), *torch.autograd.grad(y, [xi, *m.parameters()], dz))

    eager = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            on_side = step()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(eager, on_side):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    kept = x.clone()
    for seed in range(4):
        x.copy_(kept.roll(seed, 0))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
