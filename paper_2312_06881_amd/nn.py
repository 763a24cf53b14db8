"""Drop-in torch modules over libdyad.

* ``DyadLinear``: one Dyad layer, y = W x + b with W = BlockDiag(W1) +
  BlockTrans(W2) in the IT / OT / DT form (paper Sec. 2.2-2.4, Eqs. 1-16), a
  replacement for ``torch.nn.Linear``.
* ``DyadFF``: the feed-forward block fc1 -> GELU -> fc2 with both layers Dyad,
  each with its own variant if wanted (a heterogeneous mix, Sec. 4).  Unfused,
  the forward writes GELU(fc1) and stashes fc1's pre-activation in the same
  epilogue; fused, fc1 writes only the pre-activation and fc2's forward and
  weight-gradient kernels apply GELU as they stage it.  Either way the backward
  applies GELU' inside fc2's input-gradient epilogue, so the activation
  gradient is never a separate pass.

* ``stash="mx8"`` on either keeps what the backward pass reads (the layer's input,
  the pre-activation) as 8-bit microscaled blocks; the gradients see the kept values.
* ``MX4DyadLinear``, ``MX4DyadFF``: inference on fp4 weights and inputs.

* ``dropout`` / ``Dropout``, ``add_norm`` / ``AddNorm``, ``linear_cross_entropy`` /
  ``LinearCrossEntropy``: what stands around the layers in a language model.  A pre-norm
  block is ``x, a = norm(x, y)`` (the last block's output joins the stream, which is normed)
  and ``y = ff(a)``; after the last one the loss over the vocabulary, whose logits
  are never kept.

Autograd runs every pass through the C-ABI (forward, input gradient, weight and
bias gradient); there is no torch fallback and CPU tensors are rejected.
Leading input dimensions are flattened into the token dimension.  Weights
are stored as [n_dyad, ceil(out/n_dyad), ceil(in/n_dyad)] tensors, W1 the
BlockDiag and W2 the BlockTrans component; widths that n_dyad does not divide
are zero-padded (appendix, caveat on rectangular W).
"""
from __future__ import annotations

import math

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import VARIANTS, DyadError, backward_dw, backward_dx, forward, lm, mx

__all__ = ["DyadLinear", "DyadFF", "MX4DyadLinear", "MX4DyadFF", "dyad_linear", "dyad_ff", "Dropout", "AddNorm",
           "LinearCrossEntropy", "dropout", "add_norm", "linear_cross_entropy"]


def _tokens(x: torch.Tensor) -> torch.Tensor:
    if x.dim() == 2 and x.is_contiguous():
        return x
    return x.reshape(-1, x.shape[-1]).contiguous()


class _DyadLinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w1, w2, bias, variant, n_out):
        ctx.variant = variant
        ctx.has_bias = bias is not None
        ctx.save_for_backward(x, w1, w2)
        return forward(x, w1, w2, bias, variant, n_out=n_out)

    @staticmethod
    def backward(ctx, dy):
        x, w1, w2 = ctx.saved_tensors
        dy = dy.contiguous()
        dx = None
        if ctx.needs_input_grad[0]:
            dx = backward_dx(dy, w1, w2, ctx.variant, n_in=x.shape[1])
        dw1 = dw2 = db = None
        if any(ctx.needs_input_grad[1:4]):
            dw1, dw2, db = backward_dw(dy, x, w1.shape[0], ctx.variant, want_db=ctx.has_bias)
        return dx, dw1, dw2, db, None, None


def _untracked(*ts):
    """Whether no forward-mode level, functorch transform or tracer is active, and every argument
    is a plain tensor."""
    if forward_ad._current_level >= 0 or torch._C._are_functorch_transforms_active():
        return False
    if torch.compiler.is_compiling() or torch.jit.is_tracing():
        return False
    return all(t is None or type(t) in (torch.Tensor, torch.nn.Parameter) for t in ts)


def _plain(*ts):
    """Whether a call records nothing and may skip autograd: gradients are off, and it is untracked."""
    return not torch.is_grad_enabled() and _untracked(*ts)


_REFUSED = (-2, -4)   # DYAD_ERR_SHAPE, DYAD_ERR_DTYPE: no fused kernel for this layer


class _DyadFFFn(torch.autograd.Function):
    """fc1 -> GELU -> fc2.  Unfused: fc1's epilogue writes GELU(h) and stashes h.  Fused:
    fc1 writes only its pre-activation h; fc2's forward and weight-gradient kernels apply
    GELU to h as they stage it (dyad_forward_ex / dyad_backward_dw_ex), so GELU(h) is never
    written.  Both: fc2's input-gradient epilogue multiplies by GELU'(h).  A layer the fused
    kernels refuse runs unfused."""

    @staticmethod
    def forward(ctx, x, w1a, w2a, ba, w1b, w2b, bb, variants, ffn, d_out, fused):
        va, vb = variants
        y = None
        if fused:
            h = forward(x, w1a, w2a, ba, va, n_out=ffn)
            try:
                y = forward(h, w1b, w2b, bb, vb, n_out=d_out, act_in="gelu")
                a = None
            except DyadError as e:
                if e.status not in _REFUSED:
                    raise
        if y is None:
            a, h = forward(x, w1a, w2a, ba, va, act="gelu", stash_h=True, n_out=ffn)
            y = forward(a, w1b, w2b, bb, vb, n_out=d_out)
        ctx.variants = variants
        ctx.bias = (ba is not None, bb is not None)
        ctx.fused = a is None
        ctx.save_for_backward(x, h, a, w1a, w2a, ba, w1b, w2b)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, h, a, w1a, w2a, ba, w1b, w2b = ctx.saved_tensors
        va, vb = ctx.variants
        dy = dy.contiguous()
        # fc2: input gradient times GELU'(fc1 pre-activation), then its weights
        dz1 = backward_dx(dy, w1b, w2b, vb, act_in="gelu", h_in=h)
        dwb = None
        if ctx.fused:
            try:
                dwb = backward_dw(dy, h, w1b.shape[0], vb, want_db=ctx.bias[1], act_in="gelu")
            except DyadError as e:
                if e.status not in _REFUSED:
                    raise
                # this weight gradient has no fused kernel: recompute GELU(h) through fc1
                a, _ = forward(x, w1a, w2a, ba, va, act="gelu", stash_h=True, n_out=h.shape[1])
        if dwb is None:
            dwb = backward_dw(dy, a, w1b.shape[0], vb, want_db=ctx.bias[1])
        dw1b, dw2b, dbb = dwb
        # fc1
        dx = backward_dx(dz1, w1a, w2a, va, n_in=x.shape[1]) if ctx.needs_input_grad[0] else None
        dw1a, dw2a, dba = backward_dw(dz1, x, w1a.shape[0], va, want_db=ctx.bias[0])
        return dx, dw1a, dw2a, dba, dw1b, dw2b, dbb, None, None, None, None


def _parts(q):
    """The tensors of an 8-bit checkpoint, as autograd saves (and frees) them."""
    return (None, None) if q is None else (q.codes, q.scales)


def _kept(parts, like, cols):
    return mx.MXTensor._of(*parts, (like.shape[0], cols), like.dtype, "int8")


class _DyadLinearStashFn(torch.autograd.Function):
    """One layer whose input is kept in 8 bits, where a weight gradient will read it."""

    @staticmethod
    def forward(ctx, x, w1, w2, bias, variant, n_out):
        ctx.variant, ctx.n_in, ctx.has_bias = variant, x.shape[1], bias is not None
        kept = mx.quantize(x) if any(ctx.needs_input_grad[1:4]) else None
        ctx.save_for_backward(w1, w2, *_parts(kept))
        return forward(x, w1, w2, bias, variant, n_out=n_out)

    @staticmethod
    def backward(ctx, dy):
        w1, w2, *kept = ctx.saved_tensors
        dy = dy.contiguous()
        dx = backward_dx(dy, w1, w2, ctx.variant, n_in=ctx.n_in) if ctx.needs_input_grad[0] else None
        dw1 = dw2 = db = None
        if any(ctx.needs_input_grad[1:4]):
            dw1, dw2, db = mx.backward_dw(dy, _kept(kept, dy, ctx.n_in), w1.shape[0], ctx.variant, want_db=ctx.has_bias)
        return dx, dw1, dw2, db, None, None


class _DyadFFStashFn(torch.autograd.Function):
    """fc1 -> GELU -> fc2 that keeps x and fc1's pre-activation in 8 bits.  The backward pass
    takes GELU' and fc2's input from the kept pre-activation, fc1's weight gradient from the
    kept x; what nothing will read is not kept."""

    @staticmethod
    def forward(ctx, x, w1a, w2a, ba, w1b, w2b, bb, variants, ffn, d_out):
        va, vb = variants
        need = ctx.needs_input_grad
        ctx.variants, ctx.n_in, ctx.bias = variants, x.shape[1], (ba is not None, bb is not None)
        kept_x = mx.quantize(x) if any(need[1:4]) else None
        ctx.ffn = ffn
        if any(need[:7]):
            a, kept_h = mx.forward_gelu(x, w1a, w2a, ba, va, n_out=ffn)
        else:
            a, kept_h = forward(x, w1a, w2a, ba, va, act="gelu", n_out=ffn), None
        ctx.save_for_backward(w1a, w2a, w1b, w2b, *_parts(kept_x), *_parts(kept_h))
        return forward(a, w1b, w2b, bb, vb, n_out=d_out)

    @staticmethod
    def backward(ctx, dy):
        w1a, w2a, w1b, w2b, *kept = ctx.saved_tensors
        va, vb = ctx.variants
        need = ctx.needs_input_grad
        dy = dy.contiguous()
        kept_h = _kept(kept[2:], dy, ctx.ffn) if any(need[:7]) else None
        dx = dw1a = dw2a = dba = dw1b = dw2b = dbb = None
        if any(need[:4]):
            # fc2's input comes out beside the gradient through it
            dz = mx.backward_dx_gelu(dy, w1b, w2b, kept_h, vb, want_act=any(need[4:7]))
            if any(need[4:7]):
                dz, a = dz
                dw1b, dw2b, dbb = backward_dw(dy, a, w1b.shape[0], vb, want_db=ctx.bias[1])
        elif any(need[4:7]):
            dw1b, dw2b, dbb = mx.backward_dw(dy, kept_h, w1b.shape[0], vb, want_db=ctx.bias[1], act_in="gelu")
        if any(need[:4]):
            if need[0]:
                dx = backward_dx(dz, w1a, w2a, va, n_in=ctx.n_in)
            if any(need[1:4]):
                dw1a, dw2a, dba = mx.backward_dw(dz, _kept(kept[:2], dz, ctx.n_in), w1a.shape[0], va, want_db=ctx.bias[0])
        return dx, dw1a, dw2a, dba, dw1b, dw2b, dbb, None, None, None


def _check_stash(stash):
    if stash not in (None, "mx8"):
        raise ValueError("stash is None or mx8")


def _variant_pair(variant):
    pair = (variant, variant) if isinstance(variant, str) else tuple(variant)
    if len(pair) != 2 or any(v not in ("IT", "OT", "DT") for v in pair):
        raise ValueError("variant is one of IT, OT, DT, or an (fc1, fc2) pair of them")
    return pair


def dyad_linear(x, w1, w2, bias=None, variant="IT", out_features=None, stash=None):
    """Functional form of ``DyadLinear``: x [..., n_in] -> [..., n_out], where n_out is
    out_features, else bias's length, else n_dyad * bo.  stash="mx8": x is kept for the
    backward pass in 8 bits."""
    _check_stash(stash)
    D, bo, _ = w1.shape
    if out_features is None:
        out_features = bias.shape[0] if bias is not None else D * bo
    if _plain(x, w1, w2, bias):
        y = forward(_tokens(x), w1, w2, bias, variant, n_out=out_features)
    elif stash:
        y = _DyadLinearStashFn.apply(_tokens(x), w1, w2, bias, variant, out_features)
    else:
        y = _DyadLinearFn.apply(_tokens(x), w1, w2, bias, variant, out_features)
    return y.reshape(*x.shape[:-1], out_features)


def dyad_ff(x, fc1, fc2, variant="IT", ffn=None, fused=False, stash=None):
    """Functional form of ``DyadFF``; fc1 / fc2 are (W1, W2, bias) triples; variant is one
    variant or an (fc1, fc2) pair; ffn is the hidden width (default n_dyad * fc1's bo).
    The output width is x's, as the block is d -> ffn -> d.  fused: GELU applied inside
    fc2's kernels, the activation never written (see _DyadFFFn).  stash="mx8": the
    backward pass reads x and the pre-activation from 8-bit checkpoints (not with fused)."""
    _check_stash(stash)
    if stash and fused:
        raise ValueError("stash and fused exclude each other")
    d = x.shape[-1]
    if ffn is None:
        ffn = fc1[0].shape[0] * fc1[0].shape[1]
    pair = _variant_pair(variant)
    if not fused and _plain(x, *fc1, *fc2):
        # nothing to stash for a backward pass: the pre-activation is not written
        a = forward(_tokens(x), *fc1, pair[0], act="gelu", n_out=ffn)
        y = forward(a, *fc2, pair[1], n_out=d)
    elif stash:
        y = _DyadFFStashFn.apply(_tokens(x), *fc1, *fc2, pair, ffn, d)
    else:
        y = _DyadFFFn.apply(_tokens(x), *fc1, *fc2, pair, ffn, d, bool(fused))
    return y.reshape(*x.shape[:-1], d)


class DyadLinear(torch.nn.Module):
    """Dyad replacement for ``torch.nn.Linear(in_features, out_features)``.

    A width that ``n_dyad`` does not divide is zero-padded up to the next multiple
    (appendix, caveat on rectangular W); such layers run on zero-padded copies of
    their blocks from 512 tokens, and on the general kernels below.  Initialisation
    (a convenience, not part of the method): uniform in +-1/sqrt(2 * in_features /
    n_dyad), the fan-in of one output feature (two components of in_features /
    n_dyad inputs each).  ``stash="mx8"`` keeps the input in 8 bits for the backward pass.
    """

    stash = None        # of modules pickled without one

    def __init__(self, in_features, out_features, n_dyad, variant="IT", bias=True, device=None,
                 dtype=torch.bfloat16, stash=None):
        super().__init__()
        _check_stash(stash)
        self.stash = stash
        if min(in_features, out_features, n_dyad) <= 0:
            raise ValueError("widths and n_dyad must be positive")
        if variant not in ("IT", "OT", "DT"):
            raise ValueError("variant is one of IT, OT, DT")
        self.in_features, self.out_features, self.n_dyad, self.variant = in_features, out_features, n_dyad, variant
        shape = (n_dyad, -(-out_features // n_dyad), -(-in_features // n_dyad))
        kw = {"device": device, "dtype": dtype}
        self.w1 = torch.nn.Parameter(torch.empty(shape, **kw))
        self.w2 = torch.nn.Parameter(torch.empty(shape, **kw))
        self.bias = torch.nn.Parameter(torch.empty(out_features, **kw)) if bias else None
        self.reset_parameters()

    def reset_parameters(self):
        bound = 1.0 / math.sqrt(2 * self.in_features / self.n_dyad)
        with torch.no_grad():
            for p in (self.w1, self.w2, self.bias):
                if p is not None:
                    p.uniform_(-bound, bound)

    def forward(self, x):
        return dyad_linear(x, self.w1, self.w2, self.bias, self.variant, self.out_features, self.stash)

    def extra_repr(self):
        return (f"in_features={self.in_features}, out_features={self.out_features}, "
                f"n_dyad={self.n_dyad}, variant={self.variant}, bias={self.bias is not None}")


class DyadFF(torch.nn.Module):
    """Feed-forward block fc1 (d -> ffn) -> GELU -> fc2 (ffn -> d), both Dyad layers.

    ``variant`` is one of IT / OT / DT for both layers, or an (fc1, fc2) pair for a
    heterogeneous mix; ``n_dyad`` likewise may be one value or a pair.  ``fused``: fc1
    writes only its pre-activation and fc2's kernels apply GELU as they stage it.
    ``stash="mx8"``: the input and the pre-activation are kept in 8 bits for the backward
    pass (not with ``fused``)."""

    stash = None        # of modules pickled without one

    def __init__(self, d, ffn, n_dyad, variant="IT", bias=True, device=None, dtype=torch.bfloat16,
                 fused=False, stash=None):
        super().__init__()
        _check_stash(stash)
        if stash and fused:
            raise ValueError("stash and fused exclude each other")
        self.fused, self.stash = fused, stash
        va, vb = _variant_pair(variant)
        da, db = (n_dyad, n_dyad) if isinstance(n_dyad, int) else tuple(n_dyad)
        self.fc1 = DyadLinear(d, ffn, da, va, bias, device, dtype)
        self.fc2 = DyadLinear(ffn, d, db, vb, bias, device, dtype)
        self.variant = (va, vb)
        self.ffn = ffn

    def forward(self, x):
        return dyad_ff(x, (self.fc1.w1, self.fc1.w2, self.fc1.bias),
                       (self.fc2.w1, self.fc2.w2, self.fc2.bias), self.variant, self.ffn, self.fused, self.stash)


class _MX4Fn(torch.autograd.Function):
    """The fp4 product where autograd, forward mode or a tracer looks on: it has no gradient, and
    one that would have to pass through it is refused."""

    @staticmethod
    def forward(ctx, x, packed, bias, variant, n_in, n_out, n_dyad, act):
        return mx.forward(x, mx.MX4Weights(packed, variant, n_in, n_out, n_dyad), bias, act)

    @staticmethod
    def backward(ctx, dy):
        raise NotImplementedError("the fp4 product has no gradient")

    @staticmethod
    def jvp(ctx, *tangents):
        raise NotImplementedError("the fp4 product has no gradient, forward-mode ones included")


class MX4DyadLinear(torch.nn.Module):
    """A ``DyadLinear`` for inference on fp4 weights, its input quantised to fp4 within the
    call; the weights are quantised once, here.  act: "none" or "gelu".  It has no gradient:
    a backward pass or a tangent that reaches it raises.  Packed weights are as many bytes for
    every variant, so a state dict says what they are of, and loading another layer's raises."""

    def __init__(self, layer: DyadLinear, act="none"):
        super().__init__()
        if act not in ("none", "gelu"):
            raise ValueError("act is none or gelu")
        self.in_features, self.out_features, self.n_dyad = layer.in_features, layer.out_features, layer.n_dyad
        self.variant, self.act = layer.variant, act
        w = mx.quantize_weights(layer.w1.detach(), layer.w2.detach(), layer.variant, layer.in_features,
                                layer.out_features)
        self.register_buffer("packed", w.packed)
        self.register_buffer("bias", None if layer.bias is None else layer.bias.detach().clone())

    def _layout(self):
        return [mx.LAYOUT, VARIANTS[self.variant], self.in_features, self.out_features, self.n_dyad]

    def _save_to_state_dict(self, destination, prefix, keep_vars):
        super()._save_to_state_dict(destination, prefix, keep_vars)
        destination[prefix + "layout"] = torch.tensor(self._layout())

    def _load_from_state_dict(self, state_dict, prefix, local_metadata, strict, missing_keys, unexpected_keys, error_msgs):
        layout = state_dict.get(prefix + "layout")           # None: saved without it, nothing to compare
        if layout is not None and layout.tolist() != self._layout():
            error_msgs.append(f"{prefix}packed holds weights of (layout, variant, in, out, n_dyad) {layout.tolist()}, "
                              f"the module's are {self._layout()}")
            return
        super()._load_from_state_dict(state_dict, prefix, local_metadata, strict, missing_keys, unexpected_keys, error_msgs)
        if prefix + "layout" in unexpected_keys:
            unexpected_keys.remove(prefix + "layout")        # no parameter or buffer of the module

    def forward(self, x):
        t = _tokens(x)
        if _untracked(x, self.bias) and not (torch.is_grad_enabled() and x.requires_grad):
            w = mx.MX4Weights(self.packed, self.variant, self.in_features, self.out_features, self.n_dyad)
            y = mx.forward(t, w, self.bias, self.act)
        else:
            y = _MX4Fn.apply(t, self.packed, self.bias, self.variant, self.in_features, self.out_features, self.n_dyad,
                             self.act)
        return y.reshape(*x.shape[:-1], self.out_features)

    def extra_repr(self):
        return (f"in_features={self.in_features}, out_features={self.out_features}, n_dyad={self.n_dyad}, "
                f"variant={self.variant}, act={self.act}, bias={self.bias is not None}")


class MX4DyadFF(torch.nn.Module):
    """A ``DyadFF`` for inference on fp4 weights and inputs of both layers."""

    def __init__(self, block: DyadFF):
        super().__init__()
        self.fc1, self.fc2 = MX4DyadLinear(block.fc1, "gelu"), MX4DyadLinear(block.fc2)

    def forward(self, x):
        return self.fc2(self.fc1(x))


# ---- around the layers: dropout, the residual stream's norms, the loss ----------------------

def _saved_offset(offset):
    """(what autograd saves, what it does not) of an offset: a tensor's value has to be the
    forward pass's when the backward pass draws the mask again, and autograd checks that."""
    return (offset, None) if isinstance(offset, torch.Tensor) else (None, offset)


def _ready(t):
    """t contiguous and where the library takes it: gradients of slices and stacked scalars need not be."""
    if t is None:
        return None
    t = t if t.is_contiguous() else t.contiguous()
    return t.clone() if t.data_ptr() % 16 else t


class _DropoutFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, offset):
        ctx.p, ctx.seed = p, seed
        kept, ctx.offset = _saved_offset(offset)
        ctx.save_for_backward(kept)
        return lm.dropout(x, p, seed, offset)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        kept, = ctx.saved_tensors
        return lm.dropout(_ready(dy), ctx.p, ctx.seed, ctx.offset if kept is None else kept), None, None, None


def dropout(x, p, seed, offset=0, training=True):
    """x with values dropped with probability p and the others scaled; x itself when not training.  The mask
    follows from (seed, offset) and each value's row and column, and is drawn again for the gradient.  offset: a whole
    number, or a one-element int64 tensor on x's device, which a captured graph reads at every replay; between the
    passes it must not change."""
    if not training:
        return x
    x = _ready(x)
    if _plain(x):
        return lm.dropout(x, p, seed, offset)
    return _DropoutFn.apply(x, p, seed, offset)


class _AddNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, weight, bias, post_weight, post_bias, gate, call):
        h, out, stats, post_stats = call.forward(x, y, weight, bias, post_weight, post_bias, gate, True)
        ctx.call = call
        # an fp32 stream's h is read again, a bf16 one's formed again from x and y; of y only
        # its place counts where nothing reads it
        again = x.dtype is not torch.float32 and not call.x_is_h and call.norm != 0
        reads_y = again or call.post != 0 or gate is not None
        ctx.again = again
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(x if again else h, y if reads_y else None, weight, bias, post_weight, post_bias, gate, stats,
                              post_stats, call.dev)
        if h is x:
            h = x.view_as(x)
        return (h, out) if call.norm else h

    @staticmethod
    @once_differentiable
    def backward(ctx, dh, dout=None):
        if dh is None and dout is None:
            return (None,) * 8
        kept, y, weight, bias, post_weight, post_bias, gate, stats, post_stats, dev = ctx.saved_tensors
        call = ctx.call
        dh, dout = _ready(dh), _ready(dout)
        x, h = (kept, None) if ctx.again else (None, kept)
        if y is None and call.has_y:
            y = kept
        return (*call.backward(dh, dout, h, x, y, weight, bias, post_weight, post_bias, gate, stats, post_stats, dev,
                               ctx.needs_input_grad), None)


def add_norm(x, y=None, norm="layer", weight=None, bias=None, *, post_norm=None, post_weight=None, post_bias=None, gate=None,
             x_scale=1.0, y_scale=1.0, eps=1e-5, p=0.0, seed=0, offset=0, dtype=None):
    """(h, out): h = x_scale x + y_scale gate * dropout(post_norm(y)), the residual stream with a block's output,
    and out = norm(h), the next block's input.  x and y [..., n]; see ``lm.add_norm``.  out is None without a norm.
    For the backward pass an fp32 stream keeps h, a bf16 one x and y (h is formed again, without its rounding)."""
    shape = x.shape
    if y is not None and y.shape != shape:
        raise ValueError(f"x and y have one shape, got {tuple(shape)} and {tuple(y.shape)}")
    xt, yt = _ready(_tokens(x)), None if y is None else _ready(_tokens(y))
    call = lm._AddNorm(xt, yt, norm, weight, bias, post_norm, post_weight, post_bias, gate, x_scale, y_scale, eps, p, seed,
                       offset, dtype)
    if _plain(x, y, weight, bias, post_weight, post_bias, gate):
        h, out, _, _ = call.forward(xt, yt, weight, bias, post_weight, post_bias, gate, False)
    elif call.norm:
        h, out = _AddNormFn.apply(xt, yt, weight, bias, post_weight, post_bias, gate, call)
    else:
        h, out = _AddNormFn.apply(xt, yt, weight, bias, post_weight, post_bias, gate, call), None
    if xt is x:
        return h, out
    return h.reshape(shape), None if out is None else out.reshape(shape)


class _LinearCrossEntropyFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, targets, ignore_index, reduction):
        loss, lse, count = lm.linear_cross_entropy(x, weight, targets, ignore_index, reduction, keep=True)
        ctx.ignore_index, ctx.reduction = ignore_index, reduction
        ctx.save_for_backward(x, weight, targets, lse, count)
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        x, weight, targets, lse, count = ctx.saved_tensors
        dx, dw = lm.linear_cross_entropy_backward(_ready(dloss), x, weight, targets, lse, count, ctx.ignore_index,
                                                  ctx.reduction, *ctx.needs_input_grad[:2])
        return dx, dw, None, None, None


def linear_cross_entropy(x, weight, targets, ignore_index=-100, reduction="mean"):
    """Softmax cross entropy of the logits x W^T against targets, x [..., n], weight [V, n], targets [...] int64:
    float32, of targets' shape for reduction "none", else a scalar.  The logits are formed in tiles, in both
    passes, and never kept.  See ``lm.linear_cross_entropy``."""
    if targets.shape != x.shape[:-1]:
        raise ValueError(f"targets have shape {tuple(x.shape[:-1])}, got {tuple(targets.shape)}")
    xt, t = _ready(_tokens(x)), _ready(targets.reshape(-1))
    if _plain(x, weight):
        loss = lm.linear_cross_entropy(xt, weight, t, ignore_index, reduction)
    else:
        loss = _LinearCrossEntropyFn.apply(xt, weight, t, ignore_index, reduction)
    return loss.reshape(targets.shape) if reduction == "none" else loss


def _draw():
    """A whole number from torch's CPU generator, whatever the default device is."""
    return int(torch.randint(2 ** 62, (), device="cpu").item())


class Dropout(torch.nn.Module):
    """Dropout whose mask is drawn from a counter and never stored.  Every call in training draws its offset (kept in
    ``offset``) from torch's CPU generator, so torch.manual_seed makes runs repeat, and activation checkpointing, which
    restores that generator, draws the same mask when it runs the layer again.  seed: by default drawn there too (0 for a
    layer made with p = 0, which draws nothing); layers that share one still differ by their offsets.  capturable: the
    offset counts calls on the device (``calls``, with the module), so that every replay of a captured call draws
    another mask.  Such a layer needs a seed of its own (copies of it count alike), and is refused where checkpointing
    runs it again, with another count."""

    def __init__(self, p=0.1, seed=None, capturable=False, device=None):
        super().__init__()
        if not 0.0 <= p <= 1.0:
            raise ValueError(f"p is a probability, got {p}")
        self.p, self.capturable, self.offset = p, capturable, None
        self.seed = seed if seed is not None else _draw() if p or capturable else 0
        if capturable:
            self.register_buffer("calls", torch.zeros((1,), dtype=torch.int64, device=device))

    def next_offset(self):
        """The offset of the call that asks."""
        if self.capturable:
            if torch._C._current_graph_task_id() != -1:      # inside a backward pass
                raise RuntimeError("a capturable Dropout cannot be run again by activation checkpointing: its count has "
                                   "gone on, and with it the mask; capturable=False draws the same mask again")
            now = self.calls.clone()     # the backward pass draws this call's mask again
            self.calls += 1
            return now
        self.offset = _draw()
        return self.offset

    def forward(self, x):
        if not self.training or self.p == 0.0:
            return x
        return dropout(x, self.p, self.seed, self.next_offset())

    def extra_repr(self):
        return f"p={self.p}, capturable={self.capturable}"


class AddNorm(torch.nn.Module):
    """Joins a block's output with the residual stream and norms the stream for the next block:
    ``h, out = add_norm(x, y)``, or ``add_norm(x)`` before the first block.

    norm, post_norm: "layer", "rms" or None; gate: a learned scale of the block's output, one a column, from
    ``gate_init``; p: dropout of the block's output (after post_norm) in training."""

    def __init__(self, d, norm="layer", post_norm=None, gate=False, gate_init=1.0, x_scale=1.0, y_scale=1.0, eps=1e-5,
                 p=0.0, bias=True, seed=None, capturable=False, device=None, dtype=torch.bfloat16):
        super().__init__()
        for kind, what in ((norm, "norm"), (post_norm, "post_norm")):
            lm._norm_kind(kind, what)
        self.d, self.norm, self.post_norm = d, norm, post_norm
        self.x_scale, self.y_scale, self.eps = x_scale, y_scale, eps

        def vector(wanted, value):
            return torch.nn.Parameter(torch.full((d,), value, device=device, dtype=dtype)) if wanted else None

        self.weight, self.bias = vector(norm, 1.0), vector(norm == "layer" and bias, 0.0)
        self.post_weight, self.post_bias = vector(post_norm, 1.0), vector(post_norm == "layer" and bias, 0.0)
        self.gate = vector(gate, gate_init)
        self.dropout = Dropout(p, seed, capturable, device)

    def forward(self, x, y=None):
        if y is None:
            return add_norm(x, None, self.norm, self.weight, self.bias, eps=self.eps,
                            dtype=None if self.weight is None or x.dtype != torch.float32 else self.weight.dtype)
        random = {}
        if self.training and self.dropout.p:
            random = {"p": self.dropout.p, "seed": self.dropout.seed, "offset": self.dropout.next_offset()}
        return add_norm(x, y, self.norm, self.weight, self.bias, post_norm=self.post_norm, post_weight=self.post_weight,
                        post_bias=self.post_bias, gate=self.gate, x_scale=self.x_scale, y_scale=self.y_scale, eps=self.eps,
                        **random)

    def extra_repr(self):
        return f"{self.d}, norm={self.norm}, post_norm={self.post_norm}, gate={self.gate is not None}"


class LinearCrossEntropy(torch.nn.Module):
    """The last layer and the loss of a language model: softmax cross entropy of x W^T, W [vocab, d] (``weight``;
    pass the embedding's to share it).  The logits are never kept."""

    def __init__(self, d, vocab, weight=None, ignore_index=-100, reduction="mean", device=None, dtype=torch.bfloat16):
        super().__init__()
        if reduction not in lm.REDUCTIONS:
            raise ValueError("reduction is none, sum or mean")
        if weight is None:
            weight = torch.nn.Parameter(torch.empty((vocab, d), device=device, dtype=dtype).normal_(std=0.02))
        elif tuple(weight.shape) != (vocab, d):
            raise ValueError(f"weight has shape {tuple(weight.shape)}, expected {(vocab, d)}")
        self.weight, self.ignore_index, self.reduction = weight, ignore_index, reduction

    def forward(self, x, targets):
        return linear_cross_entropy(x, self.weight, targets, self.ignore_index, self.reduction)

    def extra_repr(self):
        return f"vocab={self.weight.shape[0]}, d={self.weight.shape[1]}, reduction={self.reduction}"
