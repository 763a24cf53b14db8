"""What stands around the Dyad layers of a language model: tensor-level helpers over ``dyad_dropout``,
``dyad_add_norm_*`` and ``dyad_linear_ce_*``.

* ``dropout(x, p, seed, offset)``: its mask is drawn from a counter, never stored; the gradient is
  the same call on the gradient.
* ``add_norm(x, y, ...)``, ``add_norm_backward``: h = x_scale x + y_scale gate * dropout(post(y)),
  out = norm(h), and the gradients.
* ``linear_cross_entropy(x, weight, targets, ...)``, ``linear_cross_entropy_backward``: the softmax
  cross entropy of x W^T, whose logits are never kept.

Tensors are contiguous; outputs and workspaces come from torch's allocator on the inputs' device and
every call runs on torch's current stream there.  Autograd does not see these calls; the functions
and modules in ``nn`` are what it does.
"""
from __future__ import annotations

import contextlib
import ctypes
import struct

import torch

import paper_2312_06881_amd as _dy
from . import (_check, _dtype, _ptr, _stream, AddNormArgs, AddNormGrads, CE_BACKWARD, CE_FORWARD, NORM_LAYER, NORM_NONE,
               NORM_RMS, REDUCE_MEAN, REDUCE_NONE, REDUCE_SUM)
from .mx import _bytes, _same_device

__all__ = ["dropout", "add_norm", "add_norm_backward", "linear_cross_entropy", "linear_cross_entropy_backward"]

NORMS = {None: NORM_NONE, "layer": NORM_LAYER, "rms": NORM_RMS}
REDUCTIONS = {"none": REDUCE_NONE, "sum": REDUCE_SUM, "mean": REDUCE_MEAN}


_HERE = contextlib.nullcontext()


def _on(x):
    """The launches go to x's device."""
    if not x.is_cuda:
        raise ValueError("libdyad takes device tensors")
    # (x exists, so the device runtime is up)
    return _HERE if x.get_device() == torch._C._cuda_getDevice() else torch.cuda.device(x.device)


def _random(p, seed, offset, like):
    """(p, seed, offset, device offset or None), checked."""
    p = float(p)
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"p is a probability, got {p}")
    dev = None
    if isinstance(offset, torch.Tensor):
        if offset.dtype is not torch.int64 or offset.numel() != 1:
            raise ValueError("a tensor offset is one int64")
        _same_device(like, offset)
        offset, dev = 0, offset
    if not (0 <= seed < 2 ** 64 and 0 <= offset < 2 ** 64):
        raise ValueError("seed and offset are whole numbers of 64 bits")
    return p, seed, offset, dev


def _dev(t):
    return None if t is None else _ptr(t)


def dropout(x, p, seed, offset=0):
    """x [..., cols] with values dropped with probability p (a multiple of 2^-16) and the others scaled.
    The mask follows from (seed, offset, row, column).  offset: a whole number, or a one-element int64
    tensor on x's device, read when the kernel runs."""
    p, seed, offset, dev = _random(p, seed, offset, x)
    dt, ptr = _dtype(x), _ptr(x)
    y = torch.empty_like(x)
    if x.numel():
        cols = x.shape[-1] if x.dim() else 1
        with _on(x):
            _check(_dy.dyad_dropout(x.numel() // cols, cols, dt, ptr, p, seed, offset, _dev(dev), _ptr(y), _stream(x)))
    return y


def _norm_kind(kind, what):
    if kind not in NORMS:
        raise ValueError(f"{what} is layer, rms or None")
    return NORMS[kind]


def _dtype_of(dtype):
    if dtype not in _dy._DT:
        raise TypeError(f"tensors are float32 or bfloat16, got {dtype}")
    return _dy._DT[dtype]


_HEAD = struct.Struct("=3q5i3fd2Q")     # the values and the pointers of dyad_add_norm_args
_POINTERS = struct.Struct("=12Q")
_GRADS = struct.Struct("=9Q")
assert _HEAD.size + _POINTERS.size == ctypes.sizeof(AddNormArgs) and _GRADS.size == ctypes.sizeof(AddNormGrads)


def _p(t):
    return 0 if t is None else t.data_ptr()


class _AddNorm:
    """A checked add_norm of x (or what stands for it), y and parameters, for its forward and backward calls."""

    __slots__ = ("head", "M", "n", "norm", "post", "x_type", "dtype", "device", "has_y", "x_is_h", "dev")

    def __init__(self, x, y, norm, weight, bias, post_norm, post_weight, post_bias, gate, x_scale, y_scale, eps, p, seed,
                 offset, dtype):
        M, n = x.shape
        if y is not None and y.shape != x.shape:
            raise ValueError(f"x and y have one shape, got {tuple(x.shape)} and {tuple(y.shape)}")
        if dtype is not None and y is not None and dtype != y.dtype:
            raise ValueError("out has y's dtype")
        kinds = _norm_kind(norm, "norm"), _norm_kind(post_norm, "post_norm")
        if y is None and (post_norm or gate is not None or p):
            raise ValueError("post_norm, gate and dropout are of y")
        if not norm and (weight is not None or bias is not None):
            raise ValueError("weight and bias are of the norm")
        if not post_norm and (post_weight is not None or post_bias is not None):
            raise ValueError("post_weight and post_bias are of the post norm")
        p, seed, offset, dev = _random(p, seed, offset, x)
        dtype = dtype or (x if y is None else y).dtype
        param, groups = None, 1
        for t in (weight, bias, post_weight, post_bias, gate):
            if t is None:
                continue
            if param is None:
                param = t.dtype
            elif t.dtype is not param:
                raise TypeError(f"the parameters share one dtype, got {param} and {t.dtype}")
            if t is not gate and t.shape != (n,):
                raise ValueError(f"the norms' weights have shape {(n,)}, got {tuple(t.shape)}")
            if t.device != x.device:
                _same_device(x, t)
            if not t.is_contiguous():
                raise ValueError("libdyad takes contiguous tensors")
        if gate is not None:
            groups = gate.shape[0] if gate.dim() == 2 else 1
            if gate.dim() not in (1, 2) or gate.shape[-1] != n or groups == 0 or M % groups:
                raise ValueError(f"gate is {(n,)}, or {('groups', n)} with groups dividing the {M} tokens, got "
                                 f"{tuple(gate.shape)}")
        _ptr(x), _ptr(y), _same_device(x, y)
        self.M, self.n, self.norm, self.post, self.dev = M, n, kinds[0], kinds[1], dev
        self.x_type, self.dtype, self.device, self.has_y = x.dtype, dtype, x.device, y is not None
        self.x_is_h = y is None and x_scale == 1.0
        self.head = _HEAD.pack(M, n, groups, _dtype_of(x.dtype), _dtype_of(dtype), _dtype_of(param or dtype), *kinds, x_scale,
                               y_scale, eps, p, seed, offset)

    def forward(self, x, y, weight, bias, post_weight, post_bias, gate, keep):
        """(h, out, stats, post_stats)."""
        M, n, new = self.M, self.n, torch.empty
        h = x if self.x_is_h else torch.empty_like(x)
        out = new((M, n), dtype=self.dtype, device=self.device) if self.norm else None
        stats = new((M, 2), dtype=torch.float32, device=self.device) if keep and self.norm else None
        post_stats = new((M, 2), dtype=torch.float32, device=self.device) if keep and self.post else None
        if self.norm or not self.x_is_h:
            args = self.head + _POINTERS.pack(_p(self.dev), x.data_ptr(), _p(y), _p(weight), _p(bias), _p(post_weight),
                                              _p(post_bias), _p(gate), 0 if self.x_is_h else h.data_ptr(), _p(out), _p(stats),
                                              _p(post_stats))
            with _on(x):
                _check(_dy._load().dyad_add_norm_forward(args, _stream(x)))
        return h, out, stats, post_stats

    def backward(self, dh, dout, h, x, y, weight, bias, post_weight, post_bias, gate, stats, post_stats, dev, want):
        """The gradients of x, y, weight, bias, post_weight, post_bias and gate, None where ``want`` is false.  x None: h is
        read, else it is formed again from x and y.  A y whose values nothing reads may be any tensor."""
        M, n, like = self.M, self.n, x if h is None else h
        rows = [torch.empty((M, n), dtype=t, device=self.device) if w else None
                for w, t in ((want[0], self.x_type), (want[1], self.dtype))]
        grads = rows + [torch.empty_like(t) if w and t is not None else None
                        for w, t in zip(want[2:], (weight, bias, post_weight, post_bias, gate))]
        args = self.head + _POINTERS.pack(_p(dev), _p(x), _p(y), _p(weight), _p(bias), _p(post_weight), _p(post_bias),
                                          _p(gate), _p(h), 0, _p(stats), _p(post_stats))
        g = _GRADS.pack(_p(dh), _p(dout), *map(_p, grads))
        lib = _dy._load()
        need = lib.dyad_add_norm_workspace_bytes(args, g)
        ws = torch.empty((need,), dtype=torch.uint8, device=self.device) if need else None
        with _on(like):
            _check(lib.dyad_add_norm_backward(args, g, _p(ws), need, _stream(like)))
        return grads


def add_norm(x, y=None, norm="layer", weight=None, bias=None, *, post_norm=None, post_weight=None, post_bias=None,
             gate=None, x_scale=1.0, y_scale=1.0, eps=1e-5, p=0.0, seed=0, offset=0, dtype=None, keep=False):
    """(h, out): h = x_scale x + y_scale gate * dropout(post_norm(y)), out = norm(h), of rows x, y [M, n].

    norm, post_norm: "layer", "rms" or None (no norm; out is None without one); gate [n] or [groups, n],
    row m taking gate row m // (M / groups); p, seed, offset as in ``dropout``.  h has x's type, out y's
    (without y: dtype, by default x's).  Without y and with x_scale 1, h is x itself.  keep: also the rows' statistics,
    (h, out, stats, post_stats), for ``add_norm_backward``."""
    call = _AddNorm(x, y, norm, weight, bias, post_norm, post_weight, post_bias, gate, x_scale, y_scale, eps, p, seed, offset,
                    dtype)
    res = call.forward(x, y, weight, bias, post_weight, post_bias, gate, keep)
    return res if keep else res[:2]


def add_norm_backward(dh, dout, stats, post_stats=None, x=None, y=None, norm="layer", weight=None, bias=None, *, h=None,
                      post_norm=None, post_weight=None, post_bias=None, gate=None, x_scale=1.0, y_scale=1.0, eps=1e-5,
                      p=0.0, seed=0, offset=0, dtype=None,
                      want=("x", "y", "weight", "bias", "post_weight", "post_bias", "gate")):
    """The gradients of ``add_norm`` as a dict, of what ``want`` names and the call has.  stats, post_stats: what
    add_norm(..., keep=True) returned; dh, dout: the gradients that reach h and out, either may be None; the others are
    the forward call's.  h in place of x: it is read, where with x it is formed again from x and y, which keeps a bf16
    stream's rounding of it out of the gradients."""
    like = x if x is not None else h
    if like is None or (x is not None and h is not None):
        raise ValueError("x or h")
    call = _AddNorm(like, y, norm, weight, bias, post_norm, post_weight, post_bias, gate, x_scale, y_scale, eps, p, seed, offset,
                    dtype)
    for t, kind in ((dh, like.dtype), (dout, call.dtype)):
        if t is not None and (t.shape != like.shape or t.dtype != kind):
            raise ValueError(f"a gradient has shape {tuple(like.shape)} and {kind}, got {tuple(t.shape)} and {t.dtype}")
    for s in (stats, post_stats):
        if s is not None and (s.shape != (call.M, 2) or s.dtype is not torch.float32):
            raise ValueError(f"statistics are float32 {(call.M, 2)}")
    if (norm and stats is None) or (post_norm and post_stats is None):
        raise ValueError("the statistics that add_norm(..., keep=True) returned are missing")
    if dout is not None and not norm:
        raise ValueError("there is no out without a norm")
    for t in (dh, dout, stats, post_stats):
        _ptr(t), _same_device(like, t)
    names = ("x", "y", "weight", "bias", "post_weight", "post_bias", "gate")
    there = (like, y, weight, bias, post_weight, post_bias, gate)
    got = call.backward(dh, dout, h, x, y, weight, bias, post_weight, post_bias, gate, stats, post_stats, call.dev,
                        [k in want and t is not None for k, t in zip(names, there)])
    return {k: g for k, g in zip(names, got) if g is not None}


def _loss_arguments(x, weight, targets, reduction):
    if reduction not in REDUCTIONS:
        raise ValueError("reduction is none, sum or mean")
    if x.dim() != 2 or weight.dim() != 2 or x.shape[1] != weight.shape[1]:
        raise ValueError(f"x is [M, n] and weight [V, n], got {tuple(x.shape)} and {tuple(weight.shape)}")
    if targets.shape != x.shape[:1] or targets.dtype is not torch.int64:
        raise ValueError(f"targets are int64 {tuple(x.shape[:1])}, got {targets.dtype} {tuple(targets.shape)}")
    _same_device(x, weight, targets)
    return (*x.shape, weight.shape[0], _dtype(x, weight))


def linear_cross_entropy(x, weight, targets, ignore_index=-100, reduction="mean", keep=False):
    """Softmax cross entropy of the logits x W^T, x [M, n], weight [V, n], targets [M]: float32, [M] for reduction
    "none", else a scalar ("sum", or "mean" over the tokens that count; 0 if none does).  A target that is ignore_index
    or not in 0 .. V - 1 counts for nothing.  keep: (loss, lse [M], count), for
    ``linear_cross_entropy_backward``."""
    M, n, V, dt = _loss_arguments(x, weight, targets, reduction)
    new = dict(dtype=torch.float32, device=x.device)
    loss = torch.empty((M,) if reduction == "none" else (), **new)
    lse, count = torch.empty((M,), **new), torch.empty((1,), **new)
    with _on(x):
        need = _dy.dyad_linear_ce_workspace_bytes(CE_FORWARD, M, n, V, dt)
        ws = _bytes(need, x.device) if need else None
        _check(_dy.dyad_linear_ce_forward(M, n, V, dt, _ptr(x), _ptr(weight), _ptr(targets), ignore_index,
                                          REDUCTIONS[reduction], _ptr(loss), _ptr(lse), _ptr(count), _ptr(ws), need,
                                          _stream(x)))
    return (loss, lse, count) if keep else loss


def linear_cross_entropy_backward(dloss, x, weight, targets, lse, count, ignore_index=-100, reduction="mean", want_dx=True,
                                  want_dw=True):
    """(dx, dweight) for the gradient dloss (float32, of the loss's shape); None for what is not wanted.  lse, count:
    what linear_cross_entropy(..., keep=True) returned."""
    M, n, V, dt = _loss_arguments(x, weight, targets, reduction)
    if dloss.dtype is not torch.float32 or dloss.numel() != (M if reduction == "none" else 1):
        raise ValueError("dloss is float32, of the loss's shape")
    if lse.shape != (M,) or lse.dtype is not torch.float32 or count.numel() != 1 or count.dtype is not torch.float32:
        raise ValueError("lse and count are what linear_cross_entropy(..., keep=True) returned")
    _same_device(x, dloss, lse, count)
    dx = torch.empty_like(x) if want_dx else None
    dw = torch.empty_like(weight) if want_dw else None
    with _on(x):
        need = _dy.dyad_linear_ce_workspace_bytes(CE_BACKWARD, M, n, V, dt)
        ws = _bytes(need, x.device) if need else None
        _check(_dy.dyad_linear_ce_backward(M, n, V, dt, _ptr(x), _ptr(weight), _ptr(targets), ignore_index,
                                           REDUCTIONS[reduction], _ptr(lse), _ptr(count), _ptr(dloss), _ptr(dx),
                                           _ptr(dw), _ptr(ws), need, _stream(x)))
    return dx, dw
