"""Microscaled operators without a GPU: sizes, refusals, and the reference's own grid."""
import numpy as np
import pytest
import torch

import paper_2312_06881_amd as dy
from paper_2312_06881_amd import mx
from paper_2312_06881_amd.nn import DyadFF, DyadLinear, MX4DyadLinear, dyad_ff
from tests import mx_reference as ref

FAKE = 1 << 20   # a 16-byte-aligned non-NULL address; never dereferenced by rejected calls


def test_reference_grid():
    """Ties go to the even code, large values saturate, the scale follows the largest magnitude."""
    v = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9])
    assert ref.nearest(v, "fp4")[0].tolist() == [0, 2, 2, 4, 4, 6, 6, 7]
    assert ref.nearest(np.array([0.5 / 64, 1.5 / 64, 1.999]), "int8")[0].tolist() == [0, 2, 127]
    x = np.zeros((1, 64))
    x[0, :32], x[0, 40] = 0.99, -5.0
    assert ref.scale_exponents(x, "int8").tolist() == [[-1, 2]]
    assert ref.scale_exponents(x, "fp4").tolist() == [[-3, 0]]
    assert ref.values(x, "fp4")[0, 40] == -4.0
    assert ref.quantize(np.zeros((1, 3)), "int8")[1].tolist() == [[0]]


@pytest.mark.parametrize("call", ["dyad_mx_quantize", "dyad_mx_dequantize"])
@pytest.mark.parametrize("args,code", [
    ((2, 4, 32, 1, FAKE, FAKE, FAKE), -1),
    ((-1, 4, 32, 1, FAKE, FAKE, FAKE), -1),
    ((0, 4, 32, 9, FAKE, FAKE, FAKE), -4),
    ((0, -1, 32, 1, FAKE, FAKE, FAKE), -1),
    ((0, 4, 0, 1, FAKE, FAKE, FAKE), -1),
    ((0, 1 << 31, 32, 1, FAKE, FAKE, FAKE), -1),
    ((0, 1 << 30, 1 << 30, 1, FAKE, FAKE, FAKE), -1),
    ((0, 4, 32, 1, None, FAKE, FAKE), -1),
    ((0, 4, 32, 1, FAKE, None, FAKE), -1),
    ((0, 4, 32, 1, FAKE, FAKE, None), -1),
    ((1, 4, 32, 1, FAKE + 2, FAKE, FAKE), -3),
    ((1, 4, 32, 1, FAKE, FAKE + 8, FAKE), -3),
    ((1, 4, 32, 1, FAKE, FAKE, FAKE + 1), -3),
    ((1, 0, 32, 1, None, None, None), 0),
])
def test_quantize_rejects(call, args, code):
    assert getattr(dy, call)(*args, None) == code


def test_mx4_sizes():
    # blocks of 192: two steps of 128 reduction indices, each 1 KB of codes for a fragment of 16 rows
    # and 256 bytes of scales for four of them
    assert dy.dyad_mx4_weight_bytes(dy.IT, 768, 768, 4) == 2 * 4 * 2 * (12 * 1024 + 3 * 256)
    assert dy.dyad_mx4_workspace_bytes(dy.OT, 768, 768, 4, 17) == 4 * 2 * (2 * 1024 + 256)
    assert dy.dyad_mx4_workspace_bytes(dy.DT, 768, 768, 4, 17) == 2 * 4 * 2 * (2 * 1024 + 256)
    assert dy.dyad_mx4_workspace_bytes(dy.DT, 768, 768, 4, 0) == 0
    # a few tokens of a narrow layer are quantised where they are multiplied
    assert dy.dyad_mx4_workspace_bytes(dy.DT, 768, 768, 4, 1) == 0
    assert dy.dyad_mx4_workspace_bytes(dy.DT, 770, 768, 4, 1) > 0
    assert dy.dyad_mx4_workspace_bytes(dy.DT, 768, 768, 4, 5) > 0
    assert dy.dyad_mx4_workspace_bytes(dy.OT, 768, 768, 4, 16) == 0
    assert dy.dyad_mx4_workspace_bytes(dy.OT, 3072, 768, 4, 1) > 0
    for bad in ((3, 768, 768, 4), (0, 0, 768, 4), (0, 768, 768, 0)):
        assert dy.dyad_mx4_weight_bytes(*bad) == 0 and dy.dyad_mx4_workspace_bytes(*bad, 5) == 0


@pytest.mark.parametrize("args,code", [
    (dict(variant=3), -1),
    (dict(dtype=5), -4),
    (dict(n_in=0), -1),
    (dict(M=-1), -1),
    (dict(act=2), -1),
    (dict(X=None), -1),
    (dict(Y=None), -1),
    (dict(X=FAKE + 8), -3),
    (dict(bias=FAKE + 2), -3),
    (dict(workspace=FAKE + 4), -3),
    (dict(packed=None), -5),
    (dict(packed_bytes=100), -5),
    (dict(workspace=None), -5),
    (dict(workspace_bytes=0), -5),
    (dict(variant=1, n_in=660, n_out=660, n_dyad=33), -2),
    (dict(M=0, X=None, Y=None, workspace=None, workspace_bytes=0), 0),
])
def test_mx4_forward_rejects(args, code):
    a = dict(variant=0, n_in=64, n_out=256, n_dyad=4, M=40, dtype=1, X=FAKE, packed=FAKE, packed_bytes=1 << 30, bias=None,
             act=0, Y=FAKE, workspace=FAKE, workspace_bytes=1 << 30, stream=None)
    a.update(args)
    assert dy.dyad_mx4_forward(**a) == code


@pytest.mark.parametrize("args,code", [
    (dict(variant=-1), -1), (dict(dtype=2), -4), (dict(W2=None), -1), (dict(W1=FAKE + 2), -3), (dict(packed=FAKE + 2), -3),
    (dict(packed=None), -5), (dict(packed_bytes=8), -5),
])
def test_mx4_quantize_weights_rejects(args, code):
    a = dict(variant=0, n_in=64, n_out=256, n_dyad=4, dtype=1, W1=FAKE, W2=FAKE, packed=FAKE, packed_bytes=1 << 30, stream=None)
    a.update(args)
    assert dy.dyad_mx4_quantize_weights(**a) == code


def test_mx8_passes_reject():
    shape = dict(variant=0, n_in=64, n_out=256, n_dyad=4, M=8, dtype=1)
    tail = dict(workspace=FAKE, workspace_bytes=1 << 30, stream=None)
    fwd = dict(shape, X=FAKE, W1=FAKE, W2=FAKE, bias=None, Y=FAKE, H8=FAKE, Hs=FAKE, **tail)
    dx = dict(shape, dZ=FAKE, W1=FAKE, W2=FAKE, H8=FAKE, Hs=FAKE, dX=FAKE, A=None, **tail)
    dw = dict(shape, act_in=0, dZ=FAKE, X8=FAKE, Xs=FAKE, dW1=FAKE, dW2=FAKE, dbias=None, **tail)
    for call, good, pointers, pass_ in ((dy.dyad_forward_mx8, fwd, ("X", "W1", "W2", "Y", "H8", "Hs"), dy.MX8_FORWARD),
                                        (dy.dyad_backward_dx_mx8, dx, ("dZ", "W1", "W2", "H8", "Hs", "dX"), dy.MX8_DX),
                                        (dy.dyad_backward_dw_mx8, dw, ("dZ", "X8", "Xs", "dW1", "dW2"), dy.MX8_DW)):
        for p in pointers:
            assert call(**dict(good, **{p: None})) == -1, p
            assert call(**dict(good, **{p: FAKE + 4})) == -3, p
        assert call(**dict(good, variant=7)) == -1
        assert call(**dict(good, dtype=7)) == -4
        assert call(**dict(good, M=-2)) == -1
        # fp32 always reads its checkpoint back into the workspace
        need = dy.dyad_mx8_workspace_bytes(pass_, 0, 64, 256, 4, 8, dy.F32, 0)
        assert need > 0
        assert call(**dict(good, dtype=dy.F32, workspace_bytes=need - 1)) == -5
        assert call(**dict(good, dtype=dy.F32, workspace=None)) == -5
    assert dy.dyad_backward_dw_mx8(**dict(dw, act_in=3)) == -1
    assert dy.dyad_backward_dx_mx8(**dict(dx, A=FAKE + 2)) == -3
    for call, good in ((dy.dyad_forward_mx8, fwd), (dy.dyad_backward_dx_mx8, dx)):
        assert call(**dict(good, M=0, workspace=None, workspace_bytes=0)) == 0
    assert dy.dyad_mx8_workspace_bytes(3, 0, 64, 256, 4, 8, 1, 0) == 0
    assert dy.dyad_mx8_workspace_bytes(0, 0, 64, 256, 4, 8, 1, 5) == 0
    assert dy.dyad_mx8_workspace_bytes(0, 5, 64, 256, 4, 8, 1, 0) == 0


def test_helpers_refuse():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensors"):
        mx.quantize(x)
    with pytest.raises(TypeError):
        mx.quantize(x.half())
    with pytest.raises(ValueError, match="int8 or fp4"):
        mx.quantize(x, "fp8")
    w = torch.zeros(4, 16, 16, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="one shape"):
        mx.quantize_weights(w, w[:, :8])
    with pytest.raises(ValueError, match="does not fit"):
        mx.quantize_weights(w, w, n_in=70)
    packed = mx.MX4Weights(torch.zeros(8, dtype=torch.uint8), "IT", 64, 64, 4)
    with pytest.raises(ValueError, match="columns"):
        mx.forward(x[:, :32], packed)
    with pytest.raises(ValueError, match="bias"):
        mx.forward(x, packed, torch.zeros(3, dtype=torch.bfloat16))
    kept = mx.MXTensor(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.uint8), (4, 64),
                       torch.bfloat16, "int8")
    with pytest.raises(ValueError, match="int8 MXTensor"):
        mx.backward_dw(torch.zeros(5, 64, dtype=torch.bfloat16), kept, 4)
    with pytest.raises(ValueError, match="int8 MXTensor"):
        mx.backward_dw(torch.zeros(4, 64), kept, 4)


def test_modules_refuse():
    with pytest.raises(ValueError, match="stash"):
        DyadLinear(64, 256, 4, stash="int4")
    with pytest.raises(ValueError, match="stash"):
        DyadFF(64, 256, 4, stash=True)
    with pytest.raises(ValueError, match="exclude"):
        DyadFF(64, 256, 4, fused=True, stash="mx8")
    ff = DyadFF(64, 256, 4, stash="mx8")
    with pytest.raises(ValueError, match="device tensors"):
        ff(torch.zeros(5, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="exclude"):
        dyad_ff(torch.zeros(5, 64), (ff.fc1.w1, ff.fc1.w2, None), (ff.fc2.w1, ff.fc2.w2, None), fused=True, stash="mx8")
    with pytest.raises(ValueError, match="device tensors"):
        MX4DyadLinear(DyadLinear(64, 256, 4))
    with pytest.raises(ValueError, match="act"):
        MX4DyadLinear(DyadLinear(64, 256, 4), "relu")
