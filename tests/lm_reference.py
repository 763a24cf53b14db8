"""Dropout, add_norm and the loss in 64 bits, from their definitions, with how far fp32 arithmetic may be off.

Each result comes with a magnitude: the sum of the magnitudes of what is added up to form it, a norm's unit
value u counting as |u| + r (mean|v| + |v|), since v - mean cancels.  An fp32 evaluation whose sums have depth
below 64 is within 2^-17 of that (sums over rows: 2^-15), plus half a step where it is rounded to fewer bits.
"""
import numpy as np
import torch

C, C_ROWS = 2.0 ** -17, 2.0 ** -15


def keep_mask(rows, cols, p, seed, offset):
    """(kept [rows, cols], scale), in whole-number Python and numpy."""
    octets = (cols + 7) // 8
    low = np.uint64(0xFFFFFFFF)
    o = np.arange(rows * octets, dtype=np.uint64)
    c = [o & low, o >> np.uint64(32), np.full_like(o, offset & 0xFFFFFFFF), np.full_like(o, offset >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    halves = np.stack([(w >> np.uint64(s)) & np.uint64(0xFFFF) for w in c for s in (0, 16)], 1)
    t = int(np.rint(65536 * p))
    kept = halves.reshape(rows, octets * 8)[:, :cols] >= t
    return torch.from_numpy(kept), 65536 / (65536 - t) if t < 65536 else 0.0


def philox_words(counter, key):
    """The generator on four counter words and two key words, one value at a time."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


class Unit:
    """v normed without weights: u, r = 1 / deviation, and u's magnitude."""

    def __init__(self, v, kind, eps, mag=0.0):
        m = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
        self.kind, self.mean = kind, m
        self.r = (((v - m) ** 2).mean(1, keepdim=True) + eps) ** -0.5
        self.u = (v - m) * self.r
        self.mag = self.u.abs() + self.r * (v.abs().mean(1, keepdim=True) + v.abs() + mag)

    def at(self, v):
        """The same with u taken from other values of v (as rounded to the stream's type)."""
        self.u = (v - self.mean) * self.r
        return self

    def grad(self, d, mag):
        s = d.mean(1, keepdim=True) if self.kind == "layer" else 0.0
        g = self.r * (d - s - self.u * (d * self.u).mean(1, keepdim=True))
        return g, self.r * (mag + mag.mean(1, keepdim=True) + self.mag * (mag * self.mag).mean(1, keepdim=True))


def add_norm(x, y, norm, w, b, post, pw, pb, gate, xs, ys, eps, p, seed, offset, kept_h=None, dh=None, dout=None):
    """{name: (value, magnitude, sums over rows)} of add_norm and, with gradients, its backward pass; CPU, float64
    arguments (None where the call has none).

    kept_h: h as the forward pass stored it, which is what the backward pass reads.  (Rounding the 64-bit h here
    instead would take the other neighbour wherever it lies within fp32's error of a midpoint of the stream's type,
    a whole step of that type in one value of u.)"""
    M, n = x.shape
    one = torch.ones(n, dtype=torch.float64)
    res = {}
    keep = 1.0
    if y is None:
        h, mag = xs * x, (xs * x).abs()
    else:
        z, zm = y, y.abs()
        if post:
            inner = Unit(y, post, eps)
            pw_ = one if pw is None else pw
            z = inner.u * pw_ + (0.0 if pb is None else pb)
            zm = inner.mag * pw_.abs() + (0.0 if pb is None else pb.abs())
        if p:
            kept, scale = keep_mask(M, n, p, seed, offset)
            keep = kept.double() * scale
        rows = one if gate is None else gate.reshape(-1, n).repeat_interleave(M // gate.reshape(-1, n).shape[0], 0)
        h = xs * x + ys * rows * keep * z
        mag = (xs * x).abs() + abs(ys) * rows.abs() * keep * zm
    res["h"] = (h, mag, False)
    if norm:
        outer = Unit(h, norm, eps, mag)
        w_ = one if w is None else w
        res["out"] = (outer.u * w_ + (0.0 if b is None else b), outer.mag * w_.abs() + (0.0 if b is None else b.abs()), False)
    if dh is None and dout is None:
        return res
    g, gm = torch.zeros_like(h), torch.zeros_like(h)
    if dout is not None:
        if kept_h is not None:
            outer.at(kept_h)
        g, gm = outer.grad(dout * w_, (dout * w_).abs())
        res["weight"] = ((dout * outer.u).sum(0), (dout.abs() * outer.mag).sum(0), True)
        res["bias"] = (dout.sum(0), dout.abs().sum(0), True)
    if dh is not None:
        g, gm = g + dh, gm + dh.abs()
    res["x"] = (xs * g, abs(xs) * gm, False)
    if y is None:
        return res
    dz, dm = ys * g * keep, abs(ys) * gm * keep
    if gate is not None:
        t, tm = dz * z, dm * zm
        G = gate.reshape(-1, n).shape[0]
        res["gate"] = (t.reshape(G, -1, n).sum(1).reshape(gate.shape), tm.reshape(G, -1, n).sum(1).reshape(gate.shape), True)
    dz, dm = dz * rows, dm * rows.abs()
    if post:
        res["post_weight"] = ((dz * inner.u).sum(0), (dm * inner.mag).sum(0), True)
        res["post_bias"] = (dz.sum(0), dm.sum(0), True)
        dz, dm = inner.grad(dz * pw_, dm * pw_.abs())
    res["y"] = (dz, dm, False)
    return res


def check(got, ref, what):
    """got against (value, magnitude, sums over rows)."""
    value, mag, rows = ref
    assert got.shape == value.shape, what
    g = got.detach().cpu().double()
    half = 2.0 ** -8 if got.dtype is torch.bfloat16 else 2.0 ** -24
    tol = half * value.abs() + (C_ROWS if rows else C) * mag + 1e-37
    bad = ~((g - value).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(((g - value).abs() / tol).max()))
