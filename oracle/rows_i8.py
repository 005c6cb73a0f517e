"""Linears on 8-bit integers in 64 bits: rows as codes and scales, the norms
that end in them, the product.  numpy, straight from the definitions; no code of
the library."""
import math

import numpy as np

LEAST = 127.0 * 2.0 ** -100


def quantum(y):
    """The scale of each row of y (NaN where a value is not finite)."""
    y = np.asarray(y, np.float64)
    if not y.shape[0]:
        return np.zeros(0)
    fine = np.isfinite(y).all(1)
    top = np.abs(np.where(fine[:, None], y, 0.0)).max(1)
    return np.where(fine, np.maximum(top, LEAST) / 127.0, np.nan)


def steps(y):
    """Each value in steps of its row: 127 y / m, the number that a code rounds."""
    y = np.asarray(y, np.float64)
    fine = np.isfinite(y).all(1)
    y = np.where(fine[:, None], y, 0.0)
    m = np.maximum(np.abs(y).max(1), LEAST) if y.shape[0] else np.zeros(0)
    return 127.0 * y / m[:, None]


def quantize(y):
    """(codes, scales) of rows y."""
    return np.rint(steps(y)).astype(np.int8), quantum(y)


def modulate(x, shift, scale, cu, eps):
    """LN(x) (1 + scale[r]) + shift[r], rows cu[r]..cu[r + 1] of request r."""
    x = np.asarray(x, np.float64)
    d = x - x.mean(1, keepdims=True)
    y = d / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    r = np.repeat(np.arange(len(cu) - 1), np.diff(cu))
    return y * (1.0 + np.asarray(scale, np.float64)[r]) + np.asarray(shift, np.float64)[r]


def rms(s, gain, eps):
    s = np.asarray(s, np.float64)
    return s / np.sqrt((s * s).mean(1, keepdims=True) + eps) * np.asarray(gain, np.float64)


def gelu_tanh(z):
    return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))


def sums(a, w):
    """The whole-number products, exact (below 2^53 in float64)."""
    return np.asarray(a, np.float64) @ np.asarray(w, np.float64).T


def linear(a, sa, w, sw, bias=None, epi="none", res=None, gate=None, cu=None):
    z = sums(a, w) * np.asarray(sa, np.float64)[:, None] * np.asarray(sw, np.float64)
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    if epi == "gelu":
        return gelu_tanh(z)
    if epi == "gated":
        z = z * np.asarray(gate, np.float64)[np.repeat(np.arange(len(cu) - 1), np.diff(cu))]
    return z if epi == "none" else np.asarray(res, np.float64) + z
