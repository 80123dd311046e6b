"""Plain 64-bit forms of the joint between a block and the residual stream, on
numpy arrays, with the backward pass written from the formulas.
"""
import numpy as np


def _f(x):
    return None if x is None else np.asarray(x, np.float64)


def norm(x, kind, eps):
    """(normalised rows, mean, 1 / deviation)."""
    m = x.mean(axis=1) if kind == "layer" else np.zeros(len(x))
    d = x - m[:, None]
    r = 1.0 / np.sqrt((d * d).mean(axis=1) + eps)
    return d * r[:, None], m, r


def norm_grad(q, xh, r, kind):
    out = q - xh * (q * xh).mean(axis=1)[:, None]
    if kind == "layer":
        out = out - q.mean(axis=1)[:, None]
    return out * r[:, None]


def affine(x, w, b):
    if w is not None:
        x = x * w
    return x if b is None else x + b


def gate_rows(gate, rows):
    """The gate of every row (1 where there is none)."""
    if gate is None:
        return 1.0
    g = np.atleast_2d(gate)
    return np.repeat(g, rows // len(g), axis=0)


def forward(x, y, kind="rms", post=True, w1=None, b1=None, gate=None, scale=1.0, w2=None, b2=None, eps=1e-5):
    """A dict: r, n, p, xh1, r1, m1, xh2, r2, m2."""
    x, y, w1, b1, gate, w2, b2 = (_f(t) for t in (x, y, w1, b1, gate, w2, b2))
    o = {"m1": np.zeros(len(x)), "r1": np.zeros(len(x)), "xh1": None, "p": None}
    if y is None:
        o["r"] = scale * x
    else:
        o["p"] = y
        if post:
            o["xh1"], o["m1"], o["r1"] = norm(y, kind, eps)
            o["p"] = affine(o["xh1"], w1, b1)
        o["r"] = scale * x + gate_rows(gate, len(x)) * o["p"]
    o["xh2"], o["m2"], o["r2"] = norm(o["r"], kind, eps)
    o["n"] = affine(o["xh2"], w2, b2)
    return o


def backward(dr, dn, x, y, kind="rms", post=True, w1=None, b1=None, gate=None, scale=1.0, w2=None, eps=1e-5):
    """A dict: dx, dy, dw1, db1, dw2, db2, dgate, and d (what reaches R)."""
    dr, dn, w1, gate, w2 = (_f(t) for t in (dr, dn, w1, gate, w2))
    f = forward(x, y, kind, post, w1, b1, gate, scale, w2, None, eps)
    rows = len(f["r"])
    d = np.zeros(f["r"].shape) if dr is None else dr
    o = {}
    if dn is not None:
        d = d + norm_grad(affine(dn, w2, None), f["xh2"], f["r2"], kind)
        o["dw2"], o["db2"] = (dn * f["xh2"]).sum(axis=0), dn.sum(axis=0)
    o["d"], o["dx"] = d, scale * d
    if y is None:
        return o
    e = d * gate_rows(gate, rows)
    if gate is not None:
        g = len(np.atleast_2d(gate))
        o["dgate"] = (d * f["p"]).reshape(g, rows // g, -1).sum(axis=1).reshape(gate.shape)
    if post:
        o["dw1"], o["db1"] = (e * f["xh1"]).sum(axis=0), e.sum(axis=0)
        o["dy"] = norm_grad(affine(e, w1, None), f["xh1"], f["r1"], kind)
    else:
        o["dy"] = e
    return o
