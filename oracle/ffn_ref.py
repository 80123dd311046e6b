"""Plain 64-bit forms of the operators of a transformer's feed-forward part,
on numpy arrays: layer norm, the gated feed-forward block and low-rank adapters
beside a shared projection, with the backward passes written from the
formulas.
"""
import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


def layer_norm(x, w=None, b=None, eps=1e-5):
    """(y, mean, rstd) of the rows of x."""
    x = np.asarray(x, np.float64)
    mean = x.mean(axis=1)
    var = ((x - mean[:, None]) ** 2).mean(axis=1)
    rstd = 1.0 / np.sqrt(var + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if w is not None:
        y = y * np.asarray(w, np.float64)
    if b is not None:
        y = y + np.asarray(b, np.float64)
    return y, mean, rstd


def layer_norm_backward(dy, x, w, mean, rstd):
    """(dx, dw, db) from the rows' mean and rstd."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    xh = (x - np.asarray(mean, np.float64)[:, None]) * np.asarray(rstd, np.float64)[:, None]
    p = dy if w is None else dy * np.asarray(w, np.float64)
    dx = np.asarray(rstd, np.float64)[:, None] * (
        p - p.mean(axis=1)[:, None] - xh * (p * xh).mean(axis=1)[:, None])
    return dx, (dy * xh).sum(axis=0), dy.sum(axis=0)


ACTIVATIONS = ("silu", "gelu", "gelu_tanh")


def activation(name, x):
    """(act(x), act'(x))."""
    x = np.asarray(x, np.float64)
    if name == "silu":
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-x))
        return x * s, s + x * s * (1.0 - s)
    if name == "gelu":
        cdf = 0.5 * (1.0 + _erf(x / math.sqrt(2.0)))
        return x * cdf, cdf + x * np.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)
    k = math.sqrt(2.0 / math.pi)
    t = np.tanh(k * (x + 0.044715 * x ** 3))
    return 0.5 * x * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * x * x)


def gated(x, wg, wu, act):
    """(h, gate, up): h = act(x wg) * (x wu)."""
    g, u = np.asarray(x, np.float64) @ wg, np.asarray(x, np.float64) @ wu
    return activation(act, g)[0] * u, g, u


def gated_ffn(x, wg, wu, wd, act):
    """(y, h, gate, up): y = h wd."""
    h, g, u = gated(x, wg, wu, act)
    return h @ wd, h, g, u


def gated_ffn_backward(dy, x, wg, wu, wd, g, u, h, act):
    """(dx, dwg, dwu, dwd, dgate, dup) from the saved gate, up and h."""
    a, da = activation(act, g)
    dh = dy @ wd.T
    du, dg = dh * a, dh * u * da
    return dg @ wg.T + du @ wu.T, x.T @ dg, x.T @ du, h.T @ dy, dg, du


def adapter_mm(x, w, down, up, index, scale=None, bias=None):
    """y = x w + bias + scale[a] (x down[a]^T) up[a]^T, a = index[row]; a row
    whose index is not one of the adapters has none."""
    x = np.asarray(x, np.float64)
    y = x @ np.asarray(w, np.float64)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    for i, a in enumerate(np.asarray(index).tolist()):
        if 0 <= a < len(down):
            t = np.asarray(down[a], np.float64) @ x[i]
            y[i] += (1.0 if scale is None else float(scale[a])) * (np.asarray(up[a], np.float64) @ t)
    return y
