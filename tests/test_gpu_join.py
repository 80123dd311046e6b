"""The residual joint and its backward pass on the GPU against the 64-bit forms.

Tolerances, elementwise, with e = 2^-24 (half a unit of fp32). A sum over a row is
off by at most 100 e of the sum of the terms' magnitudes (chains of 64 within a
lane, 6 across a wave, 16 across waves, some roundings of a term). Where a norm's
input t is off by dt, its differences from the mean are off by
    dd = dt + mean(dt) + 96 e mean|t| + 2 e (|t| + |m|)   (rms: dt),
and xh = d / deviation by dd / deviation + |xh| (mean(|xh| dd) / deviation + 101 e):
the second term is half the variance's relative error. From there on errors go
through each formula term by term: a product's factor times the other's error, 3 to
6 e of the terms for roundings; norm'(q) has two means, off by 100 e of their terms
and by their terms' errors. Sums over rows: chains of at most rows / 32 (a
workgroup's) + 80. Results add their rounding u |v|, u = 2^-8 (bf16), 2^-11 (fp16,
and 2^-25 where it is subnormal), e.
"""
import numpy as np
import pytest

import paper_2608_10803_amd as ac
from oracle import join_ref, mx_ref

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


def f64(x):
    return None if x is None else x.detach().double().cpu().numpy()


def view(t, rows, cols, dtype, pad=0, off=0, fill=None):
    """rows x cols view of a larger buffer filled with a canary."""
    buf = t.full(((rows + 1) * (cols + pad) + off,), 77, dtype=dtype, device="cuda")
    v = buf[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if fill is not None:
        v.copy_(fill)
    return v, buf


def untouched(v, buf):
    v.fill_(77)
    return bool((buf == 77).all())


def near(got, ref, tol, kind, label):
    tol = tol + UNIT[kind] * (np.abs(ref) + tol) + TINY[kind] + 1e-300
    bad = ~(np.abs(f64(got) - ref) <= tol)
    assert not bad.any(), (label, np.argwhere(bad)[:4], f64(got)[bad][:4], ref[bad][:4], np.max(np.abs(f64(got) - ref) / tol))


def norm_errors(v, dv, xh, m, r, layer):
    """Error of the normalised rows of v, itself off by dv."""
    d = dv + 0.0 * v
    if layer:
        d = d + d.mean(1)[:, None] + 96 * E * np.abs(v).mean(1)[:, None] + 2 * E * (np.abs(v) + np.abs(m)[:, None])
    return r[:, None] * d + np.abs(xh) * ((np.abs(xh) * d).mean(1) * r + 101 * E)[:, None]


def grad_errors(q, eq, xh, dxh, r, layer):
    """Error of norm'(q)."""
    s2 = np.abs((q * xh).mean(1))[:, None]
    ds2 = 100 * E * np.abs(q * xh).mean(1)[:, None] + (eq * np.abs(xh) + np.abs(q) * dxh).mean(1)[:, None]
    s1 = ds1 = 0.0
    if layer:
        s1 = np.abs(q.mean(1))[:, None]
        ds1 = 100 * E * np.abs(q).mean(1)[:, None] + eq.mean(1)[:, None]
    return r[:, None] * (eq + ds1 + np.abs(xh) * ds2 + dxh * s2 + dxh * ds2 + 6 * E * (np.abs(q) + s1 + np.abs(xh) * s2))


class Case:
    """Inputs of a joint on the GPU, and what the 64-bit form makes of them."""

    def __init__(self, t, rows, cols, types, norm, post, biases, groups, pad=0, off=0, scale=0.75, pre=True, y=True,
                 weights=True):
        g = t.Generator(device="cuda").manual_seed(rows * 31 + cols)
        self.rows, self.cols, self.types, self.norm, self.post = rows, cols, types, norm, post
        self.scale, self.pre, self.pad, self.off, self.t = scale, pre, pad, off, t
        rt, bt, wt = (dt(t, n) for n in types)

        def rnd(*s):
            return t.randn(*s, device="cuda", generator=g)

        def vec(mean, on=True):
            return (mean + 0.3 * rnd(cols)).to(wt) if on else None

        self.x, _ = view(t, rows, cols, rt, pad, off, 1.5 * rnd(rows, cols) + 0.4)
        self.y = view(t, rows, cols, bt, pad, off, rnd(rows, cols) - 0.2)[0] if y else None
        self.dr, _ = view(t, rows, cols, rt, pad, off, rnd(rows, cols))
        self.dn, _ = view(t, rows, cols, bt, pad, off, rnd(rows, cols))
        self.w1, self.b1 = vec(1.0, post and weights), vec(0.0, post and biases)
        self.w2, self.b2 = vec(1.0, pre and weights), vec(0.0, pre and biases)
        self.gate = view(t, groups, cols, wt, pad, off, 0.6 + 0.5 * rnd(groups, cols))[0] if groups else None
        self.groups = groups
        self.kw = dict(norm=norm, post=post, post_weight=self.w1, post_bias=self.b1, gate=self.gate, scale=scale,
                       weight=self.w2)
        self.ref = join_ref.forward(f64(self.x), f64(self.y), norm, post, f64(self.w1), f64(self.b1), f64(self.gate), scale,
                                    f64(self.w2), f64(self.b2), 1e-5)

    def forward(self, **k):
        t, c = self.t, self
        rt, bt, _ = (dt(t, n) for n in c.types)
        self.r, self.rbuf = view(t, c.rows, c.cols, rt, c.pad, c.off)
        self.n, self.nbuf = view(t, c.rows, c.cols, bt, c.pad, c.off) if c.pre else (None, None)
        self.stats = t.full((c.rows, 4), 77.0, device="cuda")
        ac.residual_norm_tensors(c.x, c.y, c.r, c.n, bias=c.b2, eps=1e-5, stats=c.stats, **c.kw, **k)

    def errors(self):
        """Errors of the normalised Y, of P, of R and of the normalised R."""
        f, layer, X = self.ref, self.norm == "layer", np.abs(self.scale * f64(self.x))
        if self.y is None:
            dp, dr = None, 2 * E * X
            dx1 = None
        else:
            dx1 = dp = 0.0 * X
            if self.post:
                dx1 = norm_errors(f64(self.y), 0.0, f["xh1"], f["m1"], f["r1"], layer)
                w = 1.0 if self.w1 is None else np.abs(f64(self.w1))
                b = 0.0 if self.b1 is None else np.abs(f64(self.b1))
                dp = dx1 * w + 3 * E * (np.abs(f["xh1"]) * w + b)
            g = np.abs(join_ref.gate_rows(f64(self.gate), self.rows))
            dr = g * dp + 3 * E * (X + g * np.abs(f["p"]))
        return dx1, dp, dr, norm_errors(f["r"], dr, f["xh2"], f["m2"], f["r2"], layer)

    def check_forward(self):
        f, (rt, bt, _) = self.ref, self.types
        _, _, dr, dx2 = self.errors()
        near(self.r, f["r"], dr, rt, "R")
        if self.pre:
            w = 1.0 if self.w2 is None else np.abs(f64(self.w2))
            b = 0.0 if self.b2 is None else np.abs(f64(self.b2))
            near(self.n, f["n"], dx2 * w + 3 * E * (np.abs(f["xh2"]) * w + b), bt, "N")
            assert untouched(self.n, self.nbuf)
        assert untouched(self.r, self.rbuf)
        st = f64(self.stats)
        for i, (k, on) in enumerate((("m1", self.post), ("r1", self.post), ("m2", self.pre), ("r2", self.pre))):
            want = f[k] if on else np.zeros(self.rows)
            if k[0] == "m":
                src = f64(self.y) if i == 0 else f["r"]
                tol = 100 * E * np.abs(src).mean(1) + (dr.mean(1) if i else 0.0) if on and self.norm == "layer" else 0.0
            else:
                xh = f["xh1"] if i == 1 else f["xh2"]
                dxh = self.errors()[0 if i == 1 else 3] if on else None
                tol = want * (100 * E + (np.abs(xh) * dxh).mean(1)) if on else 0.0
            assert (np.abs(st[:, i] - want) <= tol + 1e-300).all(), k

    def backward(self):
        t, c = self.t, self
        rt, bt, wt = (dt(t, n) for n in c.types)
        st = np.stack([c.ref[k] if on else np.zeros(c.rows)
                       for k, on in (("m1", c.post), ("r1", c.post), ("m2", c.pre), ("r2", c.pre))], 1)
        self.stats = t.from_numpy(st).float().cuda()
        self.dx, self.dxbuf = view(t, c.rows, c.cols, rt, c.pad, c.off)
        self.dy, self.dybuf = view(t, c.rows, c.cols, bt, c.pad, c.off) if c.y is not None else (None, None)

        def like(on):
            return t.full((c.cols,), 77.0, device="cuda", dtype=wt) if on else None

        # (gradients of weights that are 1 or biases that are 0 are to be had too)
        after = c.pre and c.dn is not None
        self.g = {"dw1": like(c.post), "db1": like(c.post), "dw2": like(after), "db2": like(after)}
        self.dgate, self.dgbuf = (view(t, c.groups, c.cols, wt, c.pad, c.off) if c.groups else (None, None))
        ac.residual_norm_backward_tensors(c.dr, c.dn if c.pre else None, c.x, c.y, c.stats, c.dx, c.dy, dpost_weight=c.g["dw1"],
                                          dpost_bias=c.g["db1"], dgate=c.dgate, dweight=c.g["dw2"], dbias=c.g["db2"], **c.kw)

    def check_backward(self):
        c, f, (rt, bt, wt), layer = self, self.ref, self.types, self.norm == "layer"
        dn = f64(c.dn) if c.pre else None  # (None too where it is missing)
        o = join_ref.backward(f64(c.dr), dn, f64(c.x), f64(c.y), c.norm, c.post, f64(c.w1), f64(c.b1), f64(c.gate), c.scale,
                              f64(c.w2), 1e-5)
        dx1, dp, _, dx2 = self.errors()
        chain = c.rows / 32 + 80
        eD = 2 * E * np.abs(o["d"])
        if dn is not None:
            q = dn if c.w2 is None else dn * f64(c.w2)
            eD = eD + grad_errors(q, E * np.abs(q), f["xh2"], dx2, f["r2"], layer)
            near(c.g["dw2"], o["dw2"], chain * E * np.abs(dn * f["xh2"]).sum(0) + (np.abs(dn) * dx2).sum(0), wt, "dw2")
            near(c.g["db2"], o["db2"], chain * E * np.abs(dn).sum(0), wt, "db2")
        near(c.dx, o["dx"], np.abs(c.scale) * eD, rt, "dX")
        assert untouched(c.dx, c.dxbuf)
        if c.y is None:
            return
        gate = join_ref.gate_rows(f64(c.gate), c.rows)
        e = o["d"] * gate
        eE = np.abs(gate) * eD + E * np.abs(e)
        if c.groups:
            per = c.rows // c.groups
            terms = chain * E * np.abs(o["d"] * f["p"]) + eD * np.abs(f["p"]) + (np.abs(o["d"]) + eD) * dp
            near(c.dgate, o["dgate"], terms.reshape(c.groups, per, -1).sum(1), wt, "dgate")
            assert untouched(c.dgate, c.dgbuf)
        eY = eE
        if c.post:
            near(c.g["db1"], o["db1"], chain * E * np.abs(e).sum(0) + eE.sum(0), wt, "db1")
            near(c.g["dw1"], o["dw1"], (chain * E * np.abs(e * f["xh1"]) + eE * np.abs(f["xh1"]) + (np.abs(e) + eE) * dx1).sum(0),
                 wt, "dw1")
            w = 1.0 if c.w1 is None else f64(c.w1)
            eY = grad_errors(e * w, np.abs(w) * eE + E * np.abs(e * w), f["xh1"], dx1, f["r1"], layer)
        near(c.dy, o["dy"], eY, bt, "dY")
        assert untouched(c.dy, c.dybuf)


SIZES = [(1, 1), (3, 7), (6, 8), (9, 64), (2, 511), (36, 512), (7, 513), (600, 1000), (4, 1024), (66, 1531), (3, 2048),
         (5, 2049), (1500, 4096), (18, 5000), (3, 8192), (2, 8200), (6, 16384), (3, 16389), (2, 33001)]
TYPES = [("f32", "f32", "f32"), ("bf16", "bf16", "f32"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "f32"),
         ("f32", "bf16", "bf16"), ("f16", "f16", "f16"), ("f16", "f16", "f32"), ("f32", "f16", "f16"), ("f32", "f16", "f32")]


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "%dx%d" % s)
def test_forward_backward(t, size, types):
    rows, cols = size
    pad, off = (0, 0) if cols % 3 else (5, 3)
    i = rows + cols + TYPES.index(types)
    norm = ("rms", "layer")[i % 2]
    groups = [1, rows, 0, next(g for g in (3, 2, 1) if rows % g == 0)][i // 2 % 4]
    c = Case(t, rows, cols, types, norm, True, i % 3 != 0, groups, pad, off)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("cols", [5, 300, 1000, 1500, 4000, 6000, 17000])
@pytest.mark.parametrize("shape", ["no post", "no pre", "neither", "no Y", "no weights"])
def test_parts(t, shape, cols, norm):
    rows = 24
    for groups in (0, 1, 4, 24):
        if shape == "no Y" and groups:
            continue
        c = Case(t, rows, cols, ("f32", "bf16", "f32"), norm, shape in ("no pre", "no weights"), shape != "no weights", groups,
                 pre=shape not in ("no pre", "neither"), y=shape != "no Y", weights=shape != "no weights")
        c.forward()
        c.check_forward()
        c.backward()
        c.check_backward()


@pytest.mark.parametrize("cols", [40, 600, 1536, 4096, 9000])
@pytest.mark.parametrize("rows,groups", [(1200, 1), (1200, 3), (1200, 24), (1200, 300), (1200, 600), (1200, 1200)])
def test_gates_of_many_groups(t, rows, groups, cols):
    c = Case(t, rows, cols, ("bf16", "bf16", "f32"), "rms", True, True, groups)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


def test_outputs_that_are_not_wanted(t):
    """Each gradient alone equals what it is with all the others; R, N and stats
    may stay away."""
    for cols in (700, 4096, 9000):
        c = Case(t, 90, cols, ("bf16", "bf16", "f32"), "layer", True, True, 3)
        c.forward()
        n = c.n.clone()
        n2 = t.empty_like(n)
        ac.residual_norm_tensors(c.x, c.y, None, n2, bias=c.b2, eps=1e-5, **c.kw)
        assert t.equal(n, n2)
        c.backward()
        full = dict(dpost_weight=c.g["dw1"], dpost_bias=c.g["db1"], dgate=c.dgate, dweight=c.g["dw2"], dbias=c.g["db2"])
        for name, want in full.items():
            alone = t.empty_like(want)
            ac.residual_norm_backward_tensors(c.dr, c.dn, c.x, c.y, c.stats, None, None, **{name: alone}, **c.kw)
            if name == "dgate" or c.groups == 0:
                assert t.equal(alone, want), name
            else:  # (without the gate's gradient the rows are cut otherwise: 80 + 90 / 32 additions of either)
                near(alone, f64(want), 200 * E * 90 * np.abs(f64(want)).max() + 200 * E * 90, "f32", name)
        dx, dy = t.empty_like(c.dx), t.empty_like(c.dy)
        ac.residual_norm_backward_tensors(c.dr, c.dn, c.x, c.y, c.stats, dx, None, **c.kw)
        ac.residual_norm_backward_tensors(c.dr, c.dn, c.x, c.y, c.stats, None, dy, **c.kw)
        assert t.equal(dx, c.dx) and t.equal(dy, c.dy)


@pytest.mark.parametrize("cols", [5, 300, 700, 1531, 4096, 6000, 9000])
@pytest.mark.parametrize("groups", [0, 1, 3, 90])
def test_each_gradient_alone_element_by_element(t, cols, groups):
    """A gradient asked for alone is within the bounds of one of many, elementwise (the
    rows may be cut otherwise), and so are dX and dY."""
    c = Case(t, 90, cols, ("f32", "bf16", "f32"), "layer", True, True, groups)
    c.forward()
    c.backward()
    alone = {"dpost_weight": "dw1", "dpost_bias": "db1", "dweight": "dw2", "dbias": "db2"}
    for name, key in alone.items():
        c.g[key] = t.full((cols,), 77.0, device="cuda")
        ac.residual_norm_backward_tensors(c.dr, c.dn, c.x, c.y, c.stats, None, None, **{name: c.g[key]}, **c.kw)
    if groups:
        c.dgate.fill_(77)
        ac.residual_norm_backward_tensors(c.dr, c.dn, c.x, c.y, c.stats, None, None, dgate=c.dgate, **c.kw)
    c.dx.fill_(77)
    c.dy.fill_(77)
    ac.residual_norm_backward_tensors(c.dr, c.dn, c.x, c.y, c.stats, c.dx, None, **c.kw)
    ac.residual_norm_backward_tensors(c.dr, c.dn, c.x, c.y, c.stats, None, c.dy, **c.kw)
    c.check_backward()


def test_one_gradient_alone_of_the_two(t):
    """dR or dN missing: as zeros."""
    for cols in (5, 300, 700, 1500, 4096, 6000, 9000):
        for types in (("f32", "f32", "f32"), ("bf16", "bf16", "f32")):
            for missing in ("dr", "dn"):
                c = Case(t, 40, cols, types, "rms", True, False, 2)
                c.forward()
                setattr(c, missing, None)
                c.backward()
                c.check_backward()


@pytest.mark.parametrize("cols", [5, 31, 32, 300, 777, 1531, 4096, 5001, 8190, 12000, 20001])
@pytest.mark.parametrize("types", [("f32", "bf16", "f32"), ("f16", "f16", "f16"), ("f32", "f32", "f32")], ids="-".join)
def test_codes_are_those_of_n(t, types, cols):
    c = Case(t, 21, cols, types, "rms", True, True, 1)
    c.forward()
    n = c.n.clone()
    cs, ss = ac.mxfp4_shapes(21, cols)
    want = t.empty(cs, dtype=t.uint8, device="cuda"), t.empty(ss, dtype=t.uint8, device="cuda")
    ac.mxfp4_quantize_tensors(n, *want)
    ref = mx_ref.quantize(f64(n))
    assert np.array_equal(want[0].cpu().numpy(), ref[0]) and np.array_equal(want[1].cpu().numpy(), ref[1])
    for with_n in (True, False):
        codes, cbuf = view(t, *cs, t.uint8, 3, 1)
        scales, sbuf = view(t, *ss, t.uint8, 3, 1)
        c.n.fill_(77)
        ac.residual_norm_tensors(c.x, c.y, c.r, c.n if with_n else None, bias=c.b2, eps=1e-5, codes=codes, code_scales=scales,
                                 **c.kw)
        assert t.equal(codes, want[0]) and t.equal(scales, want[1])
        assert not with_n or t.equal(c.n, n)
        assert untouched(codes, cbuf) and untouched(scales, sbuf)


@pytest.mark.parametrize("cols", [5, 512, 3000, 9001])
@pytest.mark.parametrize("groups", [0, 1, 3])
def test_backward_without_statistics(t, cols, groups):
    """No norm after the block and no gradient of the one before the next: the
    statistics are not needed."""
    r = np.random.default_rng(cols + groups)
    x, y, dr = (t.from_numpy(r.normal(size=(12, cols))).cuda().float() for _ in range(3))
    gate = t.from_numpy(r.normal(size=(groups, cols))).cuda().float() if groups else None
    dgate = None if gate is None else t.empty_like(gate)
    dx, dy = t.empty_like(x), t.empty_like(y)
    ac.residual_norm_backward_tensors(dr, None, x, y, None, dx, dy, post=False, gate=gate, scale=0.5, dgate=dgate)
    o = join_ref.backward(f64(dr), None, f64(x), f64(y), "rms", False, gate=f64(gate), scale=0.5)
    near(dx, o["dx"], 2 * E * np.abs(o["dx"]), "f32", "dX")
    near(dy, o["dy"], 2 * E * np.abs(o["dy"]), "f32", "dY")
    if groups:
        near(dgate, o["dgate"], 82 * E * np.abs(f64(dr) * f64(y)).reshape(groups, 12 // groups, -1).sum(1), "f32", "dgate")


@pytest.mark.parametrize("shape", ["both", "no norms", "no post"])
@pytest.mark.parametrize("cols", [5, 300, 1001, 1531, 4095, 8191, 15001, 20001])
def test_in_place(t, cols, shape):
    """R over X and N over Y give the bits of outputs of their own."""
    for types in (("bf16", "bf16", "f32"), ("f32", "f32", "f32")):
        c = Case(t, 70, cols, types, "layer", shape == "both", shape == "both", 1, pre=shape != "no norms")
        c.forward()
        r, n = c.r.clone(), c.n.clone() if c.pre else None
        x, y = c.x.clone(), c.y.clone()
        ac.residual_norm_tensors(x, y, x, y if c.pre else None, bias=c.b2, eps=1e-5, **c.kw)
        assert t.equal(x, r)
        if c.pre:
            assert t.equal(y, n)


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("cols", [5, 300, 1001, 1531, 4095, 8191, 15001])
def test_in_place_without_a_second_norm(t, cols, norm):
    """R over X with a norm after the block alone: a row's sums are those of Y, but no
    wave may write R where another one's last chunk, which overlaps it, has yet to
    read X."""
    rows, g = 2100, t.Generator(device="cuda").manual_seed(cols)
    for rt, bt, wt in (("bf16", "bf16", "f32"), ("f32", "f32", "f32"), ("f32", "f16", "f16")):
        x, y, gate, w, b = (t.randn(*s, device="cuda", generator=g).to(dt(t, n))
                            for s, n in (((rows, cols), rt), ((rows, cols), bt), ((70, cols), wt), ((cols,), wt), ((cols,), wt)))
        for kw in (dict(), dict(post_weight=w, post_bias=b), dict(post_weight=w, gate=gate[0]), dict(gate=gate)):
            apart, over = t.empty_like(x), x.clone()
            ac.residual_norm_tensors(x, y, apart, norm=norm, scale=0.75, **kw)
            ac.residual_norm_tensors(over, y, over, norm=norm, scale=0.75, **kw)
            assert t.equal(over, apart), (rt, bt, wt, list(kw))


def test_no_rows_clears_the_sums(t):
    e, cols = t.empty(0, 50, device="cuda"), 50
    g = [t.ones(cols, device="cuda") for _ in range(4)]
    gate, dgate = t.ones(7, cols, device="cuda"), t.ones(7, cols, device="cuda")
    st = t.empty(0, 4, device="cuda")
    ac.residual_norm_tensors(e, e, e, e, gate=gate, stats=st)
    ac.residual_norm_backward_tensors(e, e, e, e, st, e, e, gate=gate, dgate=dgate, dpost_weight=g[0], dpost_bias=g[1],
                                      dweight=g[2], dbias=g[3])
    assert not dgate.any() and not any(v.any() for v in g)


def test_non_finite_rows_stay_alone(t):
    for cols in (700, 4096, 20000):
        for norm in ("rms", "layer"):
            x, y = t.randn(6, cols, device="cuda"), t.randn(6, cols, device="cuda")
            clean = [t.empty_like(x), t.empty_like(x)]
            ac.residual_norm_tensors(x, y, *clean, norm=norm)
            x[1, 5], y[3, cols - 1] = float("nan"), float("inf")
            out = [t.empty_like(x), t.empty_like(x)]
            ac.residual_norm_tensors(x, y, *out, norm=norm)
            assert t.isnan(out[1][1]).all() and t.isnan(out[0][1]).sum() == 1 and t.isnan(out[1][3]).any()
            for i in (0, 2, 4, 5):
                assert t.equal(out[0][i], clean[0][i]) and t.equal(out[1][i], clean[1][i])


def test_zero_rows(t):
    """A row of zeros is normalised to zeros, also with eps 0 where it is not alone
    in having no deviation (0 / 0 is NaN, as in the formula)."""
    x, y = t.zeros(3, 400, device="cuda"), t.zeros(3, 400, device="cuda")
    r, n = t.empty_like(x), t.empty_like(x)
    ac.residual_norm_tensors(x, y, r, n)
    assert not r.any() and not n.any()
    ac.residual_norm_tensors(x, y, r, n, post=False, eps=0.0)
    assert not r.any() and t.isnan(n).all()


def test_same_bits_and_other_stream(t):
    c = Case(t, 1200, 1024, ("f32", "bf16", "f32"), "rms", True, True, 1)

    def both(stream):
        t.cuda.synchronize()
        with t.cuda.stream(stream):
            c.forward()
            c.backward()
        stream.synchronize()
        return [v.clone() for v in (c.r, c.n, c.dx, c.dy, c.dgate, c.g["dw1"], c.g["db1"], c.g["dw2"], c.g["db2"])]

    for p, q in zip(both(t.cuda.current_stream()), both(t.cuda.Stream())):
        assert t.equal(p, q)


def test_graph_replays(t):
    c = Case(t, 300, 2000, ("f32", "bf16", "f32"), "layer", True, True, 3)
    c.forward()
    c.backward()
    stats = t.empty(300, 4, device="cuda")

    def call():
        ac.residual_norm_tensors(c.x, c.y, c.r, c.n, bias=c.b2, stats=stats, **c.kw)
        ac.residual_norm_backward_tensors(c.dr, c.dn, c.x, c.y, stats, c.dx, c.dy, dpost_weight=c.g["dw1"],
                                          dpost_bias=c.g["db1"], dgate=c.dgate, dweight=c.g["dw2"], dbias=c.g["db2"], **c.kw)

    out = [c.r, c.n, c.dx, c.dy, c.dgate] + list(c.g.values())
    s = t.cuda.Stream()
    with t.cuda.stream(s):
        ac.adaptcore_reserve_workspace(s.cuda_stream, ac.adaptcore_residual_norm_backward_workspace(300, 2000, 3))
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph, stream=s):
        call()
    for i in range(4):
        c.x.copy_(t.randn(300, 2000, device="cuda"))
        t.cuda.synchronize()
        graph.replay()
        t.cuda.synchronize()
        got = [v.clone() for v in out]
        call()
        t.cuda.synchronize()
        for p, q in zip(got, out):
            assert t.equal(p, q), i


def test_gradients_against_differences(t):
    """The kernels' gradients along random directions against central differences
    of the kernels' own forward pass, fp32: the pass is off by some hundred e of its
    values, so with steps of 2^-6 a difference of a sum of n products is good to
    about 2^6 300 e sqrt(n) and the step's own third order, 2^-12 of its size."""
    c = Case(t, 12, 96, ("f32", "f32", "f32"), "layer", True, True, 3)
    c.forward()
    c.backward()

    def loss(**k):
        a = dict(x=c.x, y=c.y, w1=c.w1, b1=c.b1, gate=c.gate, w2=c.w2, b2=c.b2)
        a.update(k)
        r, n = t.empty(12, 96, device="cuda"), t.empty(12, 96, device="cuda")
        ac.residual_norm_tensors(a["x"], a["y"], r, n, norm="layer", post_weight=a["w1"], post_bias=a["b1"], gate=a["gate"],
                                 scale=c.scale, weight=a["w2"], bias=a["b2"], eps=1e-5)
        return float((r.double() * c.dr.double()).sum() + (n.double() * c.dn.double()).sum())

    grads = dict(x=c.dx, y=c.dy, gate=c.dgate, w1=c.g["dw1"], b1=c.g["db1"], w2=c.g["dw2"], b2=c.g["db2"])
    for name, g in grads.items():
        at = getattr(c, name)
        v = t.randn(at.shape, device="cuda")
        h = 2.0 ** -6
        d = (loss(**{name: at + h * v}) - loss(**{name: at - h * v})) / (2 * h)
        got = float((g.double() * v.double()).sum())
        size = float(g.double().norm() * v.double().norm())
        assert abs(got - d) <= 2 ** 6 * 300 * E * 12 * 96 ** 0.5 + 2.0 ** -10 * size, name


def test_refuses_tensors(t):
    x, y = t.randn(4, 40, device="cuda"), t.randn(4, 40, device="cuda")
    r, n = t.empty_like(x), t.empty_like(x)
    w = t.ones(40, device="cuda")
    st = t.empty(4, 4, device="cuda")
    for bad in (lambda: ac.residual_norm_tensors(x.double(), y, r, n), lambda: ac.residual_norm_tensors(x, y, r.half(), n),
                lambda: ac.residual_norm_tensors(x, y.half(), r, n),
                lambda: ac.residual_norm_tensors(x, y, r, n, post_weight=w, weight=w.half()),
                lambda: ac.residual_norm_tensors(x, y, r, n, stats=st.half()),
                lambda: ac.residual_norm_backward_tensors(x, n, x, y, st, r.half(), n)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: ac.residual_norm_tensors(x, y[:3], r, n), lambda: ac.residual_norm_tensors(x, y, r, n, norm="batch"),
                lambda: ac.residual_norm_tensors(x, y, r, n, gate=t.ones(3, 40, device="cuda")),
                lambda: ac.residual_norm_tensors(x, y, r, n, weight=w[:39]),
                lambda: ac.residual_norm_tensors(x, y, r, n, stats=st[:3]),
                lambda: ac.residual_norm_tensors(x, y.cpu(), r, n), lambda: ac.residual_norm_tensors(x, y, r[:, :39], n),
                lambda: ac.residual_norm_tensors(x, y, r, n, codes=t.empty(4, 32, dtype=t.uint8, device="cuda")),
                lambda: ac.residual_norm_backward_tensors(x, n, x, y, st, r, n, dgate=w),
                lambda: ac.residual_norm_backward_tensors(x, n, x, y, st[:2], r, n)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: ac.residual_norm_tensors(x, None, r, n, gate=w), lambda: ac.residual_norm_tensors(x, y, None, None),
                lambda: ac.residual_norm_tensors(x.half(), y, r.half(), n),
                lambda: ac.residual_norm_backward_tensors(None, None, x, y, st, r, n),
                lambda: ac.residual_norm_backward_tensors(x, n, x, y, None, r, n)):
        with pytest.raises(ac.AdaptCoreError):
            bad()
