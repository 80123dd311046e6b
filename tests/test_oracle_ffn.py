"""The plain 64-bit forms of the feed-forward operators: gradients against
central differences, and the identities that the definitions imply."""
import numpy as np
import pytest

from oracle import ffn_ref


def differences(f, x, h=1e-6):
    """Gradient of the scalar f at x by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        x0 = x[i]
        x[i] = x0 + h
        hi = f()
        x[i] = x0 - h
        lo = f()
        x[i] = x0
        g[i] = (hi - lo) / (2 * h)
    return g


# central differences of O(1) functions: h^2 of the third derivative (1e-12)
# and the rounding 1e-16 / h (1e-10), some terms summed
TOL = dict(rtol=1e-6, atol=1e-8)


@pytest.mark.parametrize("weights", [True, False])
def test_layer_norm_backward(weights):
    r = np.random.default_rng(1)
    x, dy = r.normal(size=(4, 7)) * 1.5 + 0.3, r.normal(size=(4, 7))
    w, b = (r.normal(size=7) + 1, r.normal(size=7)) if weights else (None, None)

    def f():
        return (ffn_ref.layer_norm(x, w, b)[0] * dy).sum()

    _, mean, rstd = ffn_ref.layer_norm(x, w, b)
    dx, dw, db = ffn_ref.layer_norm_backward(dy, x, w, mean, rstd)
    np.testing.assert_allclose(dx, differences(f, x), **TOL)
    if weights:
        np.testing.assert_allclose(dw, differences(f, w), **TOL)
        np.testing.assert_allclose(db, differences(f, b), **TOL)


def test_layer_norm_statistics():
    r = np.random.default_rng(2)
    y, mean, rstd = ffn_ref.layer_norm(r.normal(size=(5, 64)) * 3 + 2, eps=0.0)
    np.testing.assert_allclose(y.mean(axis=1), 0, atol=1e-12)
    np.testing.assert_allclose((y ** 2).mean(axis=1), 1, atol=1e-12)


@pytest.mark.parametrize("act", ffn_ref.ACTIVATIONS)
def test_activation_derivative(act):
    x = np.linspace(-6, 6, 41)
    h = 1e-5
    d = (ffn_ref.activation(act, x + h)[0] - ffn_ref.activation(act, x - h)[0]) / (2 * h)
    np.testing.assert_allclose(ffn_ref.activation(act, x)[1], d, rtol=1e-6, atol=1e-8)


@pytest.mark.parametrize("act", ffn_ref.ACTIVATIONS)
def test_gated_ffn_backward(act):
    r = np.random.default_rng(3)
    M, D, F = 3, 4, 5
    x, dy = r.normal(size=(M, D)), r.normal(size=(M, D))
    wg, wu, wd = r.normal(size=(D, F)), r.normal(size=(D, F)), r.normal(size=(F, D))

    def f():
        return (ffn_ref.gated_ffn(x, wg, wu, wd, act)[0] * dy).sum()

    _, h, g, u = ffn_ref.gated_ffn(x, wg, wu, wd, act)
    dx, dwg, dwu, dwd, _, _ = ffn_ref.gated_ffn_backward(dy, x, wg, wu, wd, g, u, h, act)
    for got, at in ((dx, x), (dwg, wg), (dwu, wu), (dwd, wd)):
        np.testing.assert_allclose(got, differences(f, at), **TOL)


def test_adapters_are_merged_weights():
    """Rows of one adapter equal the product with W + scale down^T up^T."""
    r = np.random.default_rng(4)
    x, w = r.normal(size=(6, 5)), r.normal(size=(5, 7))
    down, up, scale, bias = r.normal(size=(2, 3, 5)), r.normal(size=(2, 7, 3)), np.array([0.5, -2.0]), r.normal(size=7)
    index = np.array([0, 1, -1, 1, 2, 0])
    y = ffn_ref.adapter_mm(x, w, down, up, index, scale, bias)
    for i, a in enumerate(index):
        m = w + scale[a] * (up[a] @ down[a]).T if 0 <= a < 2 else w
        np.testing.assert_allclose(y[i], x[i] @ m + bias, rtol=1e-12, atol=1e-12)
