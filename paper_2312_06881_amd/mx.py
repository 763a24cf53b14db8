"""Microscaled Dyad operators: tensor-level helpers over the ``dyad_mx_*`` calls.

32 consecutive values of a row share a power of two and keep 8 bits (``"int8"``:
k / 64) or 4 (``"fp4"``: 0, .5, 1, 1.5, 2, 3, 4, 6); see ``include/dyad.h``.

* ``quantize(x, format)`` -> ``MXTensor``, whose ``dequantize()`` reads it back.
* ``quantize_weights(w1, w2, ...)`` -> ``MX4Weights``, and ``forward(x, weights)``:
  a Dyad layer's product on fp4 weights and inputs.
* ``forward_gelu``, ``backward_dx_gelu``, ``backward_dw``: the passes of a layer whose
  activations are checkpointed as int8 ``MXTensor``s.

Outputs and workspaces come from torch's allocator on the inputs' device and
every call runs on torch's current stream there.  Autograd does not see these calls;
the modules in ``nn`` are what it does.
"""
from __future__ import annotations

import torch

import paper_2312_06881_amd as _dy
from . import (_act, _check, _dtype, _ptr, _stream, _variant, _width, ACT_NONE, MX8_DW, MX8_DX,
               MX8_FORWARD, MX_FP4, MX_INT8)

__all__ = ["MXTensor", "MX4Weights", "quantize", "quantize_weights", "forward", "forward_gelu", "backward_dx_gelu",
           "backward_dw"]

FORMATS = {"int8": MX_INT8, "fp4": MX_FP4}
BLOCK = 32


def _bytes(n, device):
    return torch.empty((n,), dtype=torch.uint8, device=device)


def _same_device(x, *ts):
    for t in ts:
        if t is not None and t.device != x.device:
            raise ValueError(f"tensors must share one device, got {x.device} and {t.device}")


class MXTensor:
    """A tensor quantised along its last dimension: ``codes`` (int8 [rows, cols], or fp4
    pairs uint8 [rows, ceil(cols/2)]), ``scales`` uint8 [rows, ceil(cols/32)], and the
    ``shape`` and ``dtype`` of what they stand for.  Codes and scales that are not as
    many as that are refused, here and where they are read."""

    __slots__ = ("codes", "scales", "shape", "dtype", "format")

    def __init__(self, codes, scales, shape, dtype, format):
        if format not in FORMATS:
            raise ValueError("format is int8 or fp4")
        self.codes, self.scales, self.shape, self.dtype, self.format = codes, scales, torch.Size(shape), dtype, format
        self._check()

    @classmethod
    def _of(cls, codes, scales, shape, dtype, format):
        """One whose parts were made for it (what reads it checks them)."""
        q = cls.__new__(cls)
        q.codes, q.scales, q.shape, q.dtype, q.format = codes, scales, torch.Size(shape), dtype, format
        return q

    def _check(self):
        # the calls take no lengths: they read what the shape says
        codes, scales, shape = self.codes, self.scales, self.shape
        cols = shape[-1] if shape else 0
        rows = shape.numel() // cols if cols else -1
        width, kind = (cols, torch.int8) if self.format == "int8" else ((cols + 1) // 2, torch.uint8)
        if not (codes.numel() == rows * width and scales.numel() == rows * -(-cols // BLOCK) and codes.dtype is kind
                and scales.dtype is torch.uint8 and codes.device == scales.device and codes.is_contiguous()
                and scales.is_contiguous()):
            raise ValueError(f"an MXTensor in {self.format} of shape {tuple(shape)} does not have codes {codes.dtype} "
                             f"{tuple(codes.shape)} on {codes.device} and scales {scales.dtype} {tuple(scales.shape)} on "
                             f"{scales.device}")

    @property
    def nbytes(self):
        return self.codes.numel() + self.scales.numel()

    def dequantize(self, dtype=None):
        """The values, in ``dtype`` (float32 or bfloat16; default: the quantised tensor's)."""
        self._check()
        y = torch.empty(self.shape, dtype=dtype or self.dtype, device=self.codes.device)
        if y.numel():
            rows, cols = y.numel() // self.shape[-1], self.shape[-1]
            _check(_dy.dyad_mx_dequantize(FORMATS[self.format], rows, cols, _dtype(y), _ptr(self.codes),
                                          _ptr(self.scales), _ptr(y), _stream(y)))
        return y


def _empty(rows, cols, shape, dtype, format, device):
    codes = (torch.empty((rows, cols), dtype=torch.int8, device=device) if format == "int8" else
             torch.empty((rows, (cols + 1) // 2), dtype=torch.uint8, device=device))
    return MXTensor._of(codes, torch.empty((rows, -(-cols // BLOCK)), dtype=torch.uint8, device=device), shape, dtype, format)


def quantize(x, format="int8"):
    """x [..., cols] (float32 or bfloat16, contiguous) as an ``MXTensor`` in ``format``."""
    if format not in FORMATS:
        raise ValueError("format is int8 or fp4")
    dt, ptr = _dtype(x), _ptr(x)
    if x.dim() == 0 or x.shape[-1] == 0:
        raise ValueError("quantize takes rows of at least one value")
    cols = x.shape[-1]
    rows = x.numel() // cols
    q = _empty(rows, cols, x.shape, x.dtype, format, x.device)
    _check(_dy.dyad_mx_quantize(FORMATS[format], rows, cols, dt, ptr, _ptr(q.codes), _ptr(q.scales), _stream(x)))
    return q


# ---- the fp4 product --------------------------------------------------------------

LAYOUT = 1   # of packed fp4 weights (csrc/mx_internal.h), raised whenever that changes


class MX4Weights:
    """One layer's W1 and W2 in fp4, in the library's own layout (``packed``)."""

    __slots__ = ("packed", "variant", "n_in", "n_out", "n_dyad")

    def __init__(self, packed, variant, n_in, n_out, n_dyad):
        self.packed, self.variant, self.n_in, self.n_out, self.n_dyad = packed, variant, n_in, n_out, n_dyad


def quantize_weights(w1, w2, variant="IT", n_in=None, n_out=None):
    """W1, W2 [n_dyad, bo, bi] as ``MX4Weights``.  n_in, n_out default to n_dyad times the
    block sizes; smaller widths needing the same blocks are a zero-padded layer."""
    D, bo, bi = w1.shape
    if w2.shape != w1.shape:
        raise ValueError("W1 and W2 must have one shape")
    _same_device(w1, w2)
    n_in, n_out = _width(n_in, D, bi, "n_in"), _width(n_out, D, bo, "n_out")
    dt, p1, p2, v = _dtype(w1, w2), _ptr(w1), _ptr(w2), _variant(variant)
    need = _dy.dyad_mx4_weight_bytes(v, n_in, n_out, D)
    packed = _bytes(need, w1.device)
    _check(_dy.dyad_mx4_quantize_weights(v, n_in, n_out, D, dt, p1, p2, _ptr(packed), need, _stream(w1)))
    return MX4Weights(packed, variant, n_in, n_out, D)


def forward(x, weights, bias=None, act="none", workspace=None):
    """y = act(W Q(x) + b) per token, x [M, n_in]; x is quantised to fp4 within the call.
    workspace: uint8, at least dyad_mx4_workspace_bytes long (default: a new one)."""
    w = weights
    M, n_in = x.shape
    if n_in != w.n_in:
        raise ValueError(f"x has {n_in} columns, the weights {w.n_in}")
    if bias is not None and bias.shape != (w.n_out,):
        raise ValueError(f"bias has shape {tuple(bias.shape)}, the layer {w.n_out} outputs")
    _same_device(x, w.packed, bias, workspace)
    v, dt, xp = _variant(w.variant), _dtype(x, bias), _ptr(x)
    y = torch.empty((M, w.n_out), dtype=x.dtype, device=x.device)
    if workspace is None:
        need = _dy.dyad_mx4_workspace_bytes(v, n_in, w.n_out, w.n_dyad, M)
        workspace = _bytes(need, x.device) if need else None
    _check(_dy.dyad_mx4_forward(v, n_in, w.n_out, w.n_dyad, M, dt, xp, _ptr(w.packed), w.packed.numel(), _ptr(bias),
                                _act(act), _ptr(y), _ptr(workspace), 0 if workspace is None else workspace.nbytes,
                                _stream(x)))
    return y


# ---- passes over int8 checkpoints -----------------------------------------------------

def _workspace(pass_, v, n_in, n_out, D, M, dt, act_in, device):
    need = _dy.dyad_mx8_workspace_bytes(pass_, v, n_in, n_out, D, M, dt, act_in)
    return (_bytes(need, device), need) if need else (None, 0)


def _kept(q, M, cols, like):
    if q.format != "int8" or tuple(q.shape) != (M, cols) or q.dtype != like.dtype:
        raise ValueError(f"expected an int8 MXTensor of shape {(M, cols)} and {like.dtype}, got {q.format} "
                         f"{tuple(q.shape)} of {q.dtype}")
    q._check()
    _same_device(like, q.codes)


def _layer(x, w1, w2, bias=None, n_out=None):
    """Both components of one shape, the bias of the layer's width, all where x is."""
    if w2.shape != w1.shape:
        raise ValueError("W1 and W2 must have one shape")
    if bias is not None and bias.shape != (n_out,):
        raise ValueError(f"bias has shape {tuple(bias.shape)}, the layer {n_out} outputs")
    _same_device(x, w1, w2, bias)


def forward_gelu(x, w1, w2, bias=None, variant="IT", n_out=None):
    """(GELU(h), MXTensor of h) with h = W x + b, x [M, n_in]."""
    D, bo, bi = w1.shape
    M, n_in = x.shape
    _width(n_in, D, bi, "n_in")
    n_out = _width(n_out if n_out is not None or bias is None else bias.shape[0], D, bo, "n_out")
    _layer(x, w1, w2, bias, n_out)
    v, dt = _variant(variant), _dtype(x, w1, w2, bias)
    xp = _ptr(x)
    y = torch.empty((M, n_out), dtype=x.dtype, device=x.device)
    h = _empty(M, n_out, (M, n_out), x.dtype, "int8", x.device)
    ws, need = _workspace(MX8_FORWARD, v, n_in, n_out, D, M, dt, ACT_NONE, x.device)
    _check(_dy.dyad_forward_mx8(v, n_in, n_out, D, M, dt, xp, _ptr(w1), _ptr(w2), _ptr(bias), _ptr(y), _ptr(h.codes),
                                _ptr(h.scales), _ptr(ws), need, _stream(x)))
    return y, h


def backward_dx_gelu(dz, w1, w2, h, variant="IT", want_act=False):
    """(W^T dz) * GELU'(h) per token, h the kept pre-activation [M, n_in]; with want_act
    (that, GELU(h)), the latter being the layer's input."""
    D, bo, bi = w1.shape
    M, n_out = dz.shape
    n_in = _width(h.shape[1], D, bi, "n_in")
    _width(n_out, D, bo, "n_out")
    _kept(h, M, n_in, dz)
    _layer(dz, w1, w2)
    v, dt, zp = _variant(variant), _dtype(dz, w1, w2), _ptr(dz)
    dx = torch.empty((M, n_in), dtype=dz.dtype, device=dz.device)
    a = torch.empty_like(dx) if want_act else None
    ws, need = _workspace(MX8_DX, v, n_in, n_out, D, M, dt, ACT_NONE, dz.device)
    _check(_dy.dyad_backward_dx_mx8(v, n_in, n_out, D, M, dt, zp, _ptr(w1), _ptr(w2), _ptr(h.codes), _ptr(h.scales),
                                    _ptr(dx), _ptr(a), _ptr(ws), need, _stream(dz)))
    return (dx, a) if want_act else dx


def backward_dw(dz, x, n_dyad, variant="IT", want_db=True, act_in="none"):
    """(dW1, dW2, db) of a layer whose input was kept as x; db is None unless want_db.
    act_in="gelu": the layer's input is GELU of what x holds."""
    M, n_out = dz.shape
    n_in, D = x.shape[1], n_dyad
    _kept(x, M, n_in, dz)
    dt, zp, v, ai = _dtype(dz), _ptr(dz), _variant(variant), _act(act_in)
    shape = (D, -(-n_out // D), -(-n_in // D))
    dw1 = torch.empty(shape, dtype=dz.dtype, device=dz.device)
    dw2 = torch.empty(shape, dtype=dz.dtype, device=dz.device)
    db = torch.empty((n_out,), dtype=dz.dtype, device=dz.device) if want_db else None
    ws, need = _workspace(MX8_DW, v, n_in, n_out, D, M, dt, ai, dz.device)
    _check(_dy.dyad_backward_dw_mx8(v, n_in, n_out, D, M, dt, ai, zp, _ptr(x.codes), _ptr(x.scales), _ptr(dw1),
                                    _ptr(dw2), _ptr(db), _ptr(ws), need, _stream(dz)))
    return dw1, dw2, db
