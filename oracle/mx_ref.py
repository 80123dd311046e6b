"""Plain 64-bit forms of the microscaled 4-bit operators, on numpy arrays:
quantisation, the values again, the product and the gated pair of products.
"""
import numpy as np

from .ffn_ref import activation

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def shapes(rows, cols):
    n = -(-cols // 32)
    return (rows, 16 * n), (rows, n)


def quantize(x):
    """(codes, scales) of the rows of x."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    n = -(-cols // 32)
    v = np.zeros((rows, 32 * n))
    v[:, :cols] = x
    v = v.reshape(rows, n, 32)
    bad = ~np.isfinite(v).all(axis=2)
    v = np.where(bad[:, :, None], 0.0, v)
    top = np.abs(v).max(axis=2)
    _, e = np.frexp(top)  # top = m 2^e, m in [0.5, 1)
    e = np.where(top > 0, np.maximum(e - 1 - 2, -127), -127)
    a = np.abs(v) / np.exp2(e.astype(np.float64))[:, :, None]
    # the nearest level; between two, halfway: the even code
    code = np.zeros(a.shape, np.int64)
    for i in range(7):
        mid = (LEVELS[i] + LEVELS[i + 1]) / 2
        code += (a >= mid) if i % 2 else (a > mid)
    code += 8 * np.signbit(v)
    code = np.where(bad[:, :, None], 0, code).reshape(rows, 16 * n, 2)
    return (code[:, :, 0] + 16 * code[:, :, 1]).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales, cols):
    """rows x cols values of codes and scales."""
    rows, n = scales.shape
    c = np.stack((codes & 15, codes >> 4), axis=2).reshape(rows, n, 32).astype(np.int64)
    v = LEVELS[c & 7] * np.where(c & 8, -1.0, 1.0)
    unit = np.exp2(scales.astype(np.float64) - 127.0)
    unit = np.where(scales == 255, np.nan, unit)
    return (v * unit[:, :, None]).reshape(rows, 32 * n)[:, :cols]


def rounded(x):
    """The values that x's quantised form stands for."""
    return values(*quantize(x), np.asarray(x).shape[1])


def product(a, b, bias=None):
    y = a @ b.T
    return y if bias is None else y + np.asarray(bias, np.float64)


def gated(a, bg, bu, act):
    """(h, gate, up)."""
    g, u = a @ bg.T, a @ bu.T
    return activation(act, g)[0] * u, g, u
