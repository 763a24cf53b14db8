"""The microscaled formats in 64 bits on the CPU, from their definition: the nearest
value of the element grid, ties to the even code (comparison arithmetic only)."""
import numpy as np

import oracle

FP4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def scale_exponents(x, fmt):
    """E of every block of 32 along the rows of x [rows, cols] (fp64 holding fp32 values)."""
    rows, cols = x.shape
    full = np.zeros((rows, -(-cols // 32) * 32))
    full[:, :cols] = np.abs(x)
    top = full.reshape(rows, -1, 32).max(2)
    e = np.where(top > 0, np.frexp(np.where(top > 0, top, 1.0))[1] - 1, -127)
    return np.maximum(e - (2 if fmt == "fp4" else 0), -127)


def nearest(v, fmt):
    """(code magnitude, value) of v >= 0 on the element grid, saturating; a tie goes to the even code."""
    if fmt == "int8":
        code = np.minimum(np.rint(v * 64), 127)
        return code, code / 64
    d = np.abs(v[..., None] - FP4)
    best = d.min(-1, keepdims=True)
    # of two neighbours at one distance the even code
    code = np.where(d == best, np.arange(8) % 2, 9).argmin(-1)
    return code, FP4[code]


def quantize(x, fmt):
    """(signed codes, scale bytes, values) of finite x [rows, cols]."""
    E = scale_exponents(x, fmt)
    step = np.ldexp(1.0, np.repeat(E, 32, axis=1)[:, :x.shape[1]])
    code, value = nearest(np.abs(x) / step, fmt)
    return np.where(x < 0, -code, code).astype(np.int64), E + 127, np.where(x < 0, -value, value) * step


def values(x, fmt):
    return quantize(x, fmt)[2]


def mx4_forward(variant, n_in, n_out, D, X, W1, W2, bias, act):
    """Y of the fp4 product through the oracle: each component alone on the input rounded in its order."""
    bi, bo = -(-n_in // D), -(-n_out // D)
    cols = np.arange(D * bi)
    strided = (cols % bi) * D + cols // bi
    in_t, out_t = variant in ("IT", "DT"), variant in ("OT", "DT")

    def inputs(order):
        full = np.zeros((X.shape[0], D * bi))
        full[:, :n_in] = X
        r = np.zeros_like(full)
        r[:, order] = values(full[:, order].reshape(-1, bi), "fp4").reshape(X.shape[0], -1)
        return np.ascontiguousarray(r[:, :n_in])

    g, j, k = np.arange(D)[:, None, None], np.arange(bo)[None, :, None], np.arange(bi)[None, None, :]

    def weights(W, it, ot):
        real = ((k * D + g if it else g * bi + k) < n_in) & ((j * D + g if ot else g * bo + j) < n_out)
        return values(np.where(real, W, 0.0).reshape(-1, bi), "fp4").reshape(W.shape)

    zero = np.zeros((D, bo, bi))
    h = oracle.forward(variant, n_in, n_out, D, inputs(cols), weights(W1, False, False), zero, bias)
    h = h + oracle.forward(variant, n_in, n_out, D, inputs(strided if in_t else cols), zero, weights(W2, in_t, out_t))
    return oracle.gelu_array(h) if act == "gelu" else h
