"""The 4-bit operators and the joint where an offset passes 2^31, and where a launch
counts its chunks in more than one slab.

The rows repeat with a period that no tile, slab or wave divides. What a row gives
does not depend on where it lies, so every period of the outputs equals the first
one bit for bit, and the first one is that of a call on one period alone, which the
operators' other tests hold against the 64-bit forms; here it is held against them
too where that is cheap. Sums over all n periods: the terms are the same bits, so that
they and n times one period's are off by 2^-24 of the sum of the terms' magnitudes for
every addition of a chain. A workgroup of 1024 adds rows / 1024 rows and 1024 partial
rows are added, 64 in a chain: with one period's 1009 less than 2^12 for 2^21 rows.
"""
import numpy as np
import pytest

import paper_2608_10803_amd as ac
from oracle import mx_ref

pytestmark = pytest.mark.gpu

P = 1009
SLAB_CHUNKS = 2 ** 31 - 4096  # chunks of eight values that one slab counts


@pytest.fixture(scope="module")
def t():
    import torch
    assert torch.cuda.is_available()
    ac.adaptcore_init()
    yield torch
    torch.cuda.empty_cache()


def rnd(t, rows, cols, dtype, seed=0):
    g = t.Generator(device="cuda").manual_seed(seed + rows + 3 * cols)
    return t.randn(rows, cols, device="cuda", generator=g).to(dtype)


def tall(t, x0, n, extra=0):
    """n periods of x0 below each other, in a buffer with `extra` rows behind them."""
    x = t.empty(n * P + extra, x0.shape[1], device="cuda", dtype=x0.dtype)
    x[:n * P].view(n, P, -1).copy_(x0)
    return x[:n * P]


def canary(t, rows, cols, dtype):
    return t.full((rows + 1, cols), 77, device="cuda", dtype=dtype)


def periods_agree(y, first):
    n, step = y.shape[0] // P, max(1, 2 ** 28 // (P * y.shape[1]))
    v = y.view(n, P, -1)
    return all(bool((v[i:i + step] == first).all()) for i in range(0, n, step))


def codes_of(t, x):
    out = [t.empty(s, device="cuda", dtype=t.uint8) for s in ac.mxfp4_shapes(*x.shape)]
    return ac.mxfp4_quantize_tensors(x, *out)


def f64(x):
    return x.double().cpu().numpy()


def test_quantise_in_two_slabs(t):
    """Rows of one value: four chunks each, and more of them than one slab counts."""
    n = 532083
    rows = n * P
    assert 4 * rows > SLAB_CHUNKS
    x0 = rnd(t, P, 1, t.bfloat16)
    ref = mx_ref.quantize(f64(x0))
    x = tall(t, x0, n)
    codes, scales = canary(t, rows, 16, t.uint8), canary(t, rows, 1, t.uint8)
    ac.mxfp4_quantize_tensors(x, codes[:rows], scales[:rows])
    assert np.array_equal(codes[:P].cpu().numpy(), ref[0]) and np.array_equal(scales[:P].cpu().numpy(), ref[1])
    assert periods_agree(codes[:rows], codes[:P]) and periods_agree(scales[:rows], scales[:P])
    assert bool((codes[rows] == 77).all()) and bool((scales[rows] == 77).all())
    y = canary(t, rows, 1, t.bfloat16)
    ac.mxfp4_dequantize_tensors(codes[:rows], scales[:rows], y[:rows])
    assert np.array_equal(f64(y[:P]), mx_ref.values(*ref, 1))
    assert periods_agree(y[:rows], y[:P]) and bool((y[rows] == 77).all())


def test_quantise_long_columns(t):
    """A matrix stored as columns, the last ones past 2^31 elements."""
    n, cols = 33300, 70
    rows = n * P
    assert rows * cols > 2 ** 31
    x0 = rnd(t, P, cols, t.bfloat16)
    ref = mx_ref.quantize(f64(x0))
    x = t.empty(cols, rows, device="cuda", dtype=x0.dtype)
    x.view(cols, n, P).copy_(x0.t().contiguous()[:, None, :])
    codes, scales = canary(t, rows, 48, t.uint8), canary(t, rows, 3, t.uint8)
    ac.mxfp4_quantize_tensors(x.t(), codes[:rows], scales[:rows])
    assert np.array_equal(codes[:P].cpu().numpy(), ref[0]) and np.array_equal(scales[:P].cpu().numpy(), ref[1])
    assert periods_agree(codes[:rows], codes[:P]) and periods_agree(scales[:rows], scales[:P])
    assert bool((codes[rows] == 77).all()) and bool((scales[rows] == 77).all())


def test_product_quantises_in_two_slabs(t):
    """More rows of values than the launch in front of the tiles counts chunks of: they
    are quantised in a launch of their own."""
    n = 66512
    M = n * P
    assert 32 * M > SLAB_CHUNKS
    x0 = rnd(t, P, 1, t.bfloat16)
    b, sb = codes_of(t, rnd(t, 1, 1, t.bfloat16, 5))
    y = canary(t, M, 1, t.float32)
    ac.mxfp4_mm_tensors(tall(t, x0, n), b, sb, y[:M])
    ref = mx_ref.rounded(f64(x0)) @ mx_ref.values(b.cpu().numpy(), sb.cpu().numpy(), 1).T  # (one exact product)
    assert np.array_equal(f64(y[:P]), ref)
    assert periods_agree(y[:M], y[:P]) and bool((y[M] == 77).all())


@pytest.mark.parametrize("values", [False, True])
def test_product_of_many_rows(t, values):
    """Codes, values and outputs past 2^31 bytes and elements."""
    n, N, K = 2200, 1024, 2048
    M = n * P
    assert M * K // 2 > 2 ** 31 and M * N > 2 ** 31
    x0 = rnd(t, P, K, t.bfloat16)
    b, sb = codes_of(t, rnd(t, N, K, t.bfloat16, 1))
    bu, su = codes_of(t, rnd(t, N, K, t.bfloat16, 2) * 0.02)
    a0 = (x0,) if values else codes_of(t, x0)
    a = [tall(t, v, n) for v in a0]
    kw, kw0 = ({}, {}) if values else (dict(A_scales=a[1]), dict(A_scales=a0[1]))
    want = t.empty(P, N, device="cuda", dtype=t.bfloat16)
    y = canary(t, M, N, t.bfloat16)
    for call in (lambda a, y, k: ac.mxfp4_mm_tensors(a, b, sb, y, **k),
                 lambda a, y, k: ac.mxfp4_gated_mm_tensors(a, b, sb, bu, su, y, act="gelu", **k)):
        call(a[0], y[:M], kw)
        assert periods_agree(y[:M], y[:P]) and bool((y[M] == 77).all())
        # (one period alone may run on another tile: the sums in another order)
        call(a0[0], want, kw0)
        err = (y[:P].double() - want.double()).norm() / want.double().norm()
        assert float(err) <= 2.0 ** -8


@pytest.mark.parametrize("M", [1, 20, 40, 600])
def test_product_with_many_columns(t, M):
    """The right operand's codes past 2^31 bytes: few rows, and tiles."""
    n, K = 2200, 2048
    N = n * P
    assert N * K // 2 > 2 ** 31
    b0 = codes_of(t, rnd(t, P, K, t.bfloat16))
    b = [tall(t, v, n) for v in b0]
    x = rnd(t, M, K, t.bfloat16, 3)
    y, h = (t.full((M, N + 8), 77, device="cuda", dtype=t.bfloat16)[:, :N] for _ in range(2))
    ac.mxfp4_mm_tensors(x, *b, y)
    ac.mxfp4_gated_mm_tensors(x, *b, *b, h)
    X, B = mx_ref.rounded(f64(x)), mx_ref.values(b0[0].cpu().numpy(), b0[1].cpu().numpy(), K)
    ref = t.from_numpy(X @ B.T).cuda()
    for got, want in ((y, ref), (h, ref * ref * t.sigmoid(ref))):
        first = got[:, :P]
        assert float((first.double() - want).norm() / want.norm()) <= 2.0 ** -8
        assert all(bool((got[:, i:i + P] == first).all()) for i in range(0, N, P))
        assert bool((got.as_strided((M, 8), (N + 8, 1), N) == 77).all())


@pytest.mark.parametrize("cols", [5, 700, 1531, 4096, 9000])
def test_joint_of_a_long_pitch(t, cols):
    """Rows 2^29 elements apart, the matrices beside each other in them: the bits of
    contiguous ones."""
    rows, pitch = 5, 2 ** 29 + 8
    assert (rows - 1) * pitch > 2 ** 31 and 8 * cols <= pitch
    names = ["X", "Y", "dR", "dN", "R", "N", "dX", "dY"]
    buf = t.empty(rows, pitch, device="cuda", dtype=t.bfloat16)
    far = {k: buf[:, i * cols:(i + 1) * cols] for i, k in enumerate(names)}
    near = {k: rnd(t, rows, cols, t.bfloat16, i) for i, k in enumerate(names)}
    for k in names:
        far[k].copy_(near[k])
    w = [1 + 0.3 * rnd(t, 1, cols, t.float32, 20 + i).view(cols) for i in range(5)]
    cs, ss = ac.mxfp4_shapes(rows, cols)
    got = []
    for m in (near, far):
        stats = t.empty(rows, 4, device="cuda")
        g = [t.empty_like(v) for v in w]
        codes, scales = (t.empty(s, device="cuda", dtype=t.uint8) for s in (cs, ss))
        kw = dict(norm="layer", post_weight=w[0], post_bias=w[1], gate=w[2], weight=w[3])
        ac.residual_norm_tensors(m["X"], m["Y"], m["R"], m["N"], bias=w[4], stats=stats, codes=codes, code_scales=scales, **kw)
        ac.residual_norm_backward_tensors(m["dR"], m["dN"], m["X"], m["Y"], stats, m["dX"], m["dY"], dpost_weight=g[0],
                                          dpost_bias=g[1], dgate=g[2], dweight=g[3], dbias=g[4], **kw)
        got.append([m[k].clone() for k in names] + g + [stats, codes, scales])
    for i, (p, q) in enumerate(zip(*got)):
        assert t.equal(p, q), (names + ["dw1", "db1", "dgate", "dw2", "db2", "stats", "codes", "scales"])[i]


def test_joint_of_many_rows(t):
    n, cols = 2300, 1000
    rows = n * P
    assert rows * cols > 2 ** 31
    x0, y0, dr0, dn0 = (rnd(t, P, cols, t.bfloat16, i) for i in range(4))
    w = [1 + 0.3 * rnd(t, 1, cols, t.float32, 20 + i).view(cols) for i in range(3)]
    kw = dict(post_weight=w[0], gate=w[1], weight=w[2])

    def run(x, y, dr, dn):
        m = x.shape[0]
        r, v, st = t.empty_like(x), t.empty_like(x), t.empty(m, 4, device="cuda")
        codes, scales = t.empty(m, 1024, device="cuda", dtype=t.uint8)[:, :512], t.empty(m, 32, device="cuda", dtype=t.uint8)
        ac.residual_norm_tensors(x, y, r, v, stats=st, codes=codes, code_scales=scales, **kw)
        yield r, v, st, scales
        yield (codes.contiguous(),)
        g = [t.empty_like(u) for u in w]
        ac.residual_norm_backward_tensors(dr, dn, x, y, st, r, v, dpost_weight=g[0], dgate=g[1], dweight=g[2], **kw)
        yield r, v
        yield g

    one = [[v.clone() for v in part] for part in run(x0, y0, dr0, dn0)]
    # the terms' magnitudes in one period, from its rounded outputs (a unit of 2^-8 each)
    r, _, st, _ = (v.double() for v in one[0])
    dx, xh1, xh2 = one[2][0].double(), y0.double() * st[:, 1:2], r * st[:, 3:4]
    terms = [(dx * w[1] * xh1).abs().sum(0), (dx * xh1 * w[0]).abs().sum(0), (dn0.double() * xh2).abs().sum(0)]
    assert rows // 1024 + 64 + P < 2 ** 12
    for part, want in zip(run(*(tall(t, v, n) for v in (x0, y0, dr0, dn0))), one):
        if want[0].dim() == 1:
            for g, u, m in zip(part, want, terms):
                assert bool(((g.double() - n * u.double()).abs() <= 2.0 ** -12 * n * 1.02 * m).all())
        else:
            assert all(periods_agree(v, u) for v, u in zip(part, want))
