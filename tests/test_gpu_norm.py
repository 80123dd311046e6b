"""Layer norm and its backward pass on the GPU against the 64-bit forms.

Tolerances. With e = 2^-24 (half a unit of fp32) a sum's error is at most
e * S * sum|terms|, S the longest chain of additions: at most 64 within a lane
(eight chunks of eight), 6 across a wave, 16 across waves: S = 96. The mean m is
then within 96 e mean|x| and x^ = (x - m) r within

    dxh = r (96 e mean|x| + 2 e |x|) + 100 e |x^|

(the second term: r's own error, half that of its variance, and two
roundings). y adds two roundings, and the one to its type, u |y|, half a unit in
the last of p significant bits: u = 2^-8 (bf16, p = 8), 2^-11 (fp16, p = 11, and
2^-25 where it is subnormal), e.

The backward pass reads m and r as given: x^ is within 3 e (|x| + |m|) r, the
row sums within 100 e of the sums of absolute values; its column sums add a
chain of rows / blocks, then of the partial rows: at most rows / 256 + 80.
"""
import numpy as np
import pytest

import paper_2608_10803_amd as ac
from oracle import ffn_ref

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
UNIT = {"f32": E, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}


@pytest.fixture(scope="module")
def t():
    import torch
    assert torch.cuda.is_available()
    ac.adaptcore_init()
    return torch


def dt(t, name):
    return {"f32": t.float32, "bf16": t.bfloat16, "f16": t.float16}[name]


def rows_view(t, rows, cols, dtype, pad, offset, fill=None):
    """rows x cols view of a larger buffer (pitch cols + pad, first element
    `offset` in), and the buffer; filled with a canary."""
    buf = t.full(((rows + 1) * (cols + pad) + offset,), 777.0, dtype=dtype, device="cuda")
    v = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if fill is not None:
        v.copy_(fill)
    return v, buf


def f64(x):
    return x.detach().double().cpu().numpy()


def outside_untouched(t, view, buf):
    n = view.numel()
    return int((buf == 777.0).sum()) >= buf.numel() - n and bool((buf[-(view.stride(0)):] == 777.0).all())


SIZES = [(1, 1), (3, 7), (5, 8), (9, 64), (2, 511), (33, 512), (7, 513), (600, 1000), (4, 1024), (65, 1531), (3, 2048),
         (5, 2049), (1500, 4096), (17, 5000), (3, 8192), (2, 8200), (5, 16384), (3, 16389), (2, 32768), (3, 33001)]


@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16")],
                         ids="-".join)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "%dx%d" % s)
def test_forward_backward(t, size, types):
    rows, cols = size
    xt, wt = types
    pad, off = (0, 0) if cols % 3 else (5, 3)
    g = t.Generator(device="cuda").manual_seed(rows * 7 + cols)

    def rnd(*s):
        return t.randn(*s, device="cuda", generator=g)

    x, _ = rows_view(t, rows, cols, dt(t, xt), pad, off, rnd(rows, cols) * 1.5 + 0.7)
    dy, _ = rows_view(t, rows, cols, dt(t, xt), pad, off, rnd(rows, cols))
    w, b = (1 + 0.3 * rnd(cols)).to(dt(t, wt)), rnd(cols).to(dt(t, wt))
    y, ybuf = rows_view(t, rows, cols, dt(t, xt), pad, off)
    dx, dxbuf = rows_view(t, rows, cols, dt(t, xt), pad, off)
    mean, rstd = t.empty(rows, device="cuda"), t.empty(rows, device="cuda")
    dw, db = t.empty(cols, device="cuda", dtype=w.dtype), t.empty(cols, device="cuda", dtype=w.dtype)
    ac.layer_norm_tensors(x, w, b, y, eps=1e-5, mean=mean, rstd=rstd)
    assert outside_untouched(t, y, ybuf)
    X, W, B, DY = f64(x), f64(w), f64(b), f64(dy)
    ry, rm, rr = ffn_ref.layer_norm(X, W, B, 1e-5)
    xh = (X - rm[:, None]) * rr[:, None]
    dm = 96 * E * np.abs(X).mean(1)
    assert (np.abs(f64(mean) - rm) <= dm + 2 * E * np.abs(rm)).all()
    # r: half the variance's relative error (its chain, and the mean's error squared)
    assert (np.abs(f64(rstd) - rr) <= rr * (100 * E + dm ** 2 * rr ** 2)).all()
    dxh = rr[:, None] * (dm[:, None] + 2 * E * np.abs(X)) + (100 * E + (dm * rr)[:, None] ** 2) * np.abs(xh)
    tol = dxh * np.abs(W) + 3 * E * (np.abs(xh * W) + np.abs(B))
    tol = tol + UNIT[xt] * (np.abs(ry) + tol) + TINY[xt]
    assert (np.abs(f64(y) - ry) <= tol).all(), np.max(np.abs(f64(y) - ry) / tol)

    m32, r32 = t.from_numpy(rm).float().cuda(), t.from_numpy(rr).float().cuda()
    ac.layer_norm_backward_tensors(dy, x, w, m32, r32, dx, dweight=dw, dbias=db)
    assert outside_untouched(t, dx, dxbuf)
    M, R = f64(m32), f64(r32)
    rdx, rdw, rdb = ffn_ref.layer_norm_backward(DY, X, W, M, R)
    xh = (X - M[:, None]) * R[:, None]
    exh = 3 * E * (np.abs(X) + np.abs(M)[:, None]) * R[:, None]
    p = np.abs(DY * W)
    s1 = 100 * E * p.mean(1)[:, None]
    s2v = np.abs((DY * W * xh).mean(1))[:, None]
    s2 = 100 * E * (p * np.abs(xh)).mean(1)[:, None] + (p * exh).mean(1)[:, None]
    tol = R[:, None] * (5 * E * p + s1 + np.abs(xh) * s2 + exh * s2v + 5 * E * (np.abs(xh) * s2v))
    tol = tol + UNIT[xt] * (np.abs(rdx) + tol) + TINY[xt]
    assert (np.abs(f64(dx) - rdx) <= tol).all(), np.max(np.abs(f64(dx) - rdx) / tol)
    chain = rows / 256 + 80
    for got, ref, mag, extra in ((dw, rdw, (np.abs(DY) * np.abs(xh)).sum(0), (np.abs(DY) * exh).sum(0)),
                                 (db, rdb, np.abs(DY).sum(0), 0.0)):
        tol = chain * E * mag + extra
        tol = tol + UNIT[wt] * (np.abs(ref) + tol) + TINY[wt] + 1e-300
        assert (np.abs(f64(got) - ref) <= tol).all(), np.max(np.abs(f64(got) - ref) / tol)


def test_no_weights(t):
    x, dy = t.randn(37, 300, device="cuda"), t.randn(37, 300, device="cuda")
    y, dx = t.empty_like(x), t.empty_like(x)
    mean, rstd = t.empty(37, device="cuda"), t.empty(37, device="cuda")
    ac.layer_norm_tensors(x, None, None, y, mean=mean, rstd=rstd)
    ac.layer_norm_backward_tensors(dy, x, None, mean, rstd, dx)
    ry, rm, rr = ffn_ref.layer_norm(f64(x))
    # values of order one: the bounds above come to about 300 units
    np.testing.assert_allclose(f64(y), ry, rtol=400 * E, atol=400 * E)
    np.testing.assert_allclose(f64(dx), ffn_ref.layer_norm_backward(f64(dy), f64(x), None, rm, rr)[0], rtol=1000 * E,
                               atol=1000 * E)
    db = t.empty(300, device="cuda")
    ac.layer_norm_backward_tensors(dy, x, None, mean, rstd, dx, dbias=db)
    np.testing.assert_allclose(f64(db), f64(dy).sum(0), rtol=0, atol=100 * E * 37 * 4)


def test_no_rows_clears_weight_gradients(t):
    e = t.empty(0, 50, device="cuda")
    dw, db = t.ones(50, device="cuda"), t.ones(50, device="cuda")
    none = t.empty(0, device="cuda")
    ac.layer_norm_tensors(e, None, None, e)
    ac.layer_norm_backward_tensors(e, e, None, none, none, e, dweight=dw, dbias=db)
    assert not dw.any() and not db.any()


def test_non_finite_rows_stay_alone(t):
    for cols in (700, 4096, 40000):
        x = t.randn(6, cols, device="cuda")
        clean = t.empty_like(x)
        ac.layer_norm_tensors(x, None, None, clean)
        x[1, 5], x[3, cols - 1] = float("nan"), float("inf")
        y = t.empty_like(x)
        ac.layer_norm_tensors(x, None, None, y)
        assert t.isnan(y[1]).all() and t.isnan(y[3]).all()
        for i in (0, 2, 4, 5):
            assert t.equal(y[i], clean[i])


def test_large_mean(t):
    """A mean of 3000 deviations: the deviations keep their digits."""
    x = (t.randn(16, 2000, device="cuda") + 3000.0)
    y = t.empty_like(x)
    ac.layer_norm_tensors(x, None, None, y)
    ry, _, _ = ffn_ref.layer_norm(f64(x))
    # the mean's error (96 e 3000) against a deviation of one
    assert np.abs(f64(y) - ry).max() <= 110 * E * 3000


def test_same_bits_and_other_stream(t):
    x, dy = t.randn(3000, 1024, device="cuda").bfloat16(), t.randn(3000, 1024, device="cuda").bfloat16()
    w = t.ones(1024, device="cuda")

    def both(stream):
        y, dx = t.empty_like(x), t.empty_like(x)
        m, r = t.empty(3000, device="cuda"), t.empty(3000, device="cuda")
        dw, db = t.empty(1024, device="cuda"), t.empty(1024, device="cuda")
        with t.cuda.stream(stream):
            ac.layer_norm_tensors(x, w, None, y, mean=m, rstd=r)
            ac.layer_norm_backward_tensors(dy, x, w, m, r, dx, dweight=dw, dbias=db)
        stream.synchronize()
        return y, dx, dw, db

    t.cuda.synchronize()
    a, b = both(t.cuda.current_stream()), both(t.cuda.Stream())
    for p, q in zip(a, b):
        assert t.equal(p, q)


def test_graph_replays(t):
    """A captured forward and backward pass, with eager work between the
    replays, equals the eager result every time."""
    x, dy = t.randn(500, 2000, device="cuda"), t.randn(500, 2000, device="cuda")
    w = t.rand(2000, device="cuda")
    out = [t.empty_like(x), t.empty_like(x), t.empty(2000, device="cuda"), t.empty(2000, device="cuda")]
    m, r = t.empty(500, device="cuda"), t.empty(500, device="cuda")

    def call():
        ac.layer_norm_tensors(x, w, None, out[0], mean=m, rstd=r)
        ac.layer_norm_backward_tensors(dy, x, w, m, r, out[1], dweight=out[2], dbias=out[3])

    s = t.cuda.Stream()
    with t.cuda.stream(s):
        ac.adaptcore_reserve_workspace(s.cuda_stream, ac.adaptcore_layer_norm_backward_workspace(500, 2000))
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph, stream=s):
        call()
    for i in range(4):
        x.copy_(t.randn(500, 2000, device="cuda"))
        t.cuda.synchronize()
        graph.replay()
        t.cuda.synchronize()
        got = [o.clone() for o in out]
        call()
        t.cuda.synchronize()
        for p, q in zip(got, out):
            assert t.equal(p, q), i


def test_refuses_tensors(t):
    x = t.randn(4, 8, device="cuda")
    y = t.empty_like(x)
    for bad in (lambda: ac.layer_norm_tensors(x.double(), None, None, y),
                lambda: ac.layer_norm_tensors(x, None, None, y.bfloat16()),
                lambda: ac.layer_norm_tensors(x, t.ones(8, device="cuda"), t.ones(8, device="cuda").half(), y)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: ac.layer_norm_tensors(x, None, None, y[:3]),
                lambda: ac.layer_norm_tensors(x.t().contiguous().t(), None, None, y),
                lambda: ac.layer_norm_tensors(x, t.ones(7, device="cuda"), None, y),
                lambda: ac.layer_norm_tensors(x.cpu(), None, None, y),
                lambda: ac.layer_norm_tensors(x, t.ones(16, device="cuda")[::2], None, y),
                lambda: ac.layer_norm_tensors(x, None, None, y, mean=t.empty(3, device="cuda")),
                lambda: ac.layer_norm_backward_tensors(x, x, None, None, None, y)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("size", [(5, 1), (40, 7), (300, 512), (65, 1531), (900, 2048), (9, 5000), (33, 16384), (4, 16389),
                                  (70, 33001)], ids=lambda s: "%dx%d" % s)
def test_dx_in_place(t, size):
    """dX over dY and dX over X give the bits of a pass into its own buffer,
    the weight gradients too."""
    rows, cols = size
    for dtype in ("f32", "bf16"):
        x, dy = t.randn(rows, cols, device="cuda").to(dt(t, dtype)), t.randn(rows, cols, device="cuda").to(dt(t, dtype))
        w, y, dx = t.randn(cols, device="cuda"), t.empty_like(x), t.empty_like(x)
        m, r = t.empty(rows, device="cuda"), t.empty(rows, device="cuda")
        ac.layer_norm_tensors(x, w, None, y, mean=m, rstd=r)
        dw, db = t.empty(cols, device="cuda"), t.empty(cols, device="cuda")
        ac.layer_norm_backward_tensors(dy, x, w, m, r, dx, dweight=dw, dbias=db)
        for over in ("dy", "x"):
            a, b = dy.clone(), x.clone()
            out = a if over == "dy" else b
            dw2, db2 = t.empty(cols, device="cuda"), t.empty(cols, device="cuda")
            ac.layer_norm_backward_tensors(a, b, w, m, r, out, dweight=dw2, dbias=db2)
            assert t.equal(out, dx) and t.equal(dw2, dw) and t.equal(db2, db), (dtype, over)
