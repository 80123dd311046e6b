"""The gated feed-forward block and its backward pass on the GPU against the
64-bit formulas.

Tolerances. e = 2^-24, u = 2^-8 (bf16), 2^-11 (fp16): half a unit in the last
place. A product of depth K is summed in fp32 by at most K additions, so it is
within K e sum|a b| of the exact one; one rounding to 16 bits adds u |value|
(fp16: 2^-25 where it is subnormal). Every stage is held against the 64-bit
formula on what that stage read:

    gate, up    D e sum|x w|, one rounding
    H           |act'| <= 1.2: 1.2 dg |up| + |act| du + 16 e |h| (the
                activation's own arithmetic: exp, reciprocal, erf to a few
                units), one rounding
    Y           from the H written: F e sum|h wd|, one rounding
    dU, dG      (kept inside) dh = D e sum|dy wd|; |act| dh + u|dU| + 16 e |dU|,
                |up act'| dh + u|dG| + 16 e |dH up|
    dX, dW..    their products' sums over those errors, K e sum|a b|, one
                rounding

These are worst cases. Roundings are independent, so the 2-norm of a whole
output's error is also held to 3 u of the output's (each of at most five
roundings on the way contributes at most u / sqrt(3) of it), plus the fp32 sums'
share, below u.
"""
import pytest

import paper_2608_10803_amd as ac
from oracle import ffn_ref

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


@pytest.fixture(scope="module")
def t():
    import torch
    assert torch.cuda.is_available()
    ac.adaptcore_init()
    return torch


def act64(t, name, x):
    """(act, act') in 64 bits."""
    import math
    if name == "silu":
        s = t.sigmoid(x)
        return x * s, s * (1 + x * (1 - s))
    if name == "gelu":
        c = 0.5 * t.special.erfc(-x / math.sqrt(2))
        return x * c, c + x * t.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    th = t.tanh(k * (x + 0.044715 * x ** 3))
    return 0.5 * x * (1 + th), 0.5 * (1 + th) + 0.5 * x * (1 - th * th) * k * (1 + 3 * 0.044715 * x * x)


def test_activations_agree(t):
    x = t.linspace(-8, 8, 200, dtype=t.float64)
    for name in ffn_ref.ACTIVATIONS:
        for a, b in zip(act64(t, name, x), ffn_ref.activation(name, x.numpy())):
            assert abs(a.numpy() - b).max() < 1e-12


class Problem:
    """Inputs and canaried outputs of one block. layout: "r" or "c" for the
    up-projections, then for the down-projection; pad: elements added to every
    pitch; off: first element of every matrix within its buffer."""

    def __init__(self, t, M, D, F, dtype=None, layout="cc", act="silu", pad=0, off=0, seed=0, grads=None):
        self.t, self.M, self.D, self.F, self.act = t, M, D, F, act
        self.dt = dtype or t.bfloat16
        self.u = 2.0 ** -8 if self.dt == t.bfloat16 else 2.0 ** -11
        self.tiny = 0.0 if self.dt == t.bfloat16 else 2.0 ** -25
        self.g = t.Generator(device="cuda").manual_seed(seed + M + 3 * D + 5 * F)
        self.pad, self.off = pad, off
        self.bufs = []
        self.x = self.mat(M, D, 1.0)
        self.dy = self.mat(M, D, max(M, 1) ** -0.5)
        self.wg = self.weight(D, F, layout[0], max(D, 1) ** -0.5)
        self.wu = self.weight(D, F, layout[0], max(D, 1) ** -0.5)
        self.wd = self.weight(F, D, layout[1], max(F, 1) ** -0.5)
        gt = grads or self.dt
        self.gt = gt
        self.h, self.gate, self.up, self.y, self.dx = (self.mat(*s) for s in ((M, F), (M, F), (M, F), (M, D), (M, D)))
        self.dwg, self.dwu = (self.weight(D, F, layout[0], dt=gt) for _ in range(2))
        self.dwd = self.weight(F, D, layout[1], dt=gt)

    def mat(self, rows, cols, scale=None, dt=None):
        t = self.t
        ld = cols + self.pad
        buf = t.full((rows * ld + self.off + 64,), 555.0, dtype=dt or self.dt, device="cuda")
        v = buf[self.off:self.off + rows * ld].view(rows, ld)[:, :cols]
        if scale is not None:
            v.copy_(t.randn(rows, cols, device="cuda", generator=self.g) * scale)
        else:
            self.bufs.append((buf, v))
        return v

    def weight(self, rows, cols, layout, scale=None, dt=None):
        return self.mat(cols, rows, scale, dt).t() if layout == "c" else self.mat(rows, cols, scale, dt)

    def forward(self, save=True):
        kw = dict(gate=self.gate, up=self.up) if save else {}
        return ac.gated_ffn_tensors(self.x, self.wg, self.wu, self.wd, self.h, self.y, act=self.act, **kw)

    def backward(self, **kw):
        a = dict(dX=self.dx, dWg=self.dwg, dWu=self.dwu, dWd=self.dwd)
        a.update(kw)
        ac.gated_ffn_backward_tensors(self.dy, self.x, self.wg, self.wu, self.wd, self.gate, self.up, self.h,
                                      act=self.act, **a)

    def near(self, name, got, ref, tol, dt=None, count=1):
        """Every element within tol and one rounding; the norm within 3 u."""
        t = self.t
        f32 = (dt or self.dt) == t.float32
        u, tiny = (E, 0.0) if f32 else (self.u, self.tiny)
        got = got.double()
        assert t.isfinite(got).all(), name
        tol = tol + u * (ref.abs() + tol) + tiny + 1e-30
        worst = ((got - ref).abs() / tol).max().item() if got.numel() else 0.0
        assert worst <= 1.0, (name, worst)
        if ref.numel() >= 1000:
            rel = ((got - ref).norm() / ref.norm()).item()
            assert rel <= 3 * self.u, (name, rel)

    def check_forward(self, saved=True):
        t, F = self.t, self.F
        x, wg, wu, wd = (v.double() for v in (self.x, self.wg, self.wu, self.wd))
        g, u = x @ wg, x @ wu
        dg, du = (self.D * E * (x.abs() @ w.abs()) for w in (wg, wu))
        if saved:
            self.near("gate", self.gate, g, dg)
            self.near("up", self.up, u, du)
        a, _ = act64(t, self.act, g)
        h = a * u
        self.near("h", self.h, h, 1.2 * dg * u.abs() + a.abs() * du + 1.2 * dg * du + 16 * E * (a * u).abs()
                  + 16 * E * u.abs())
        hk = self.h.double()
        self.near("y", self.y, hk @ wd, F * E * (hk.abs() @ wd.abs()))
        self.untouched()

    def check_backward(self, dx=True, up=True, down=True):
        t = self.t
        x, wg, wu, wd, dy, g, u, h = (v.double() for v in (self.x, self.wg, self.wu, self.wd, self.dy, self.gate,
                                                           self.up, self.h))
        a, d = act64(t, self.act, g)
        dh = dy @ wd.t()
        ddh = self.D * E * (dy.abs() @ wd.t().abs())
        du, dg = dh * a, dh * u * d
        edu = a.abs() * ddh + (self.u + 32 * E) * du.abs() + 16 * E * dh.abs() + self.tiny
        edg = (u * d).abs() * ddh + (self.u + 16 * E) * dg.abs() + 16 * E * (dh * u).abs() + self.tiny
        sdu, sdg = du.abs() + edu, dg.abs() + edg
        if dx:
            ref = dg @ wg.t() + du @ wu.t()
            tol = edg @ wg.t().abs() + edu @ wu.t().abs() + 2 * self.F * E * (sdg @ wg.t().abs() + sdu @ wu.t().abs())
            self.near("dx", self.dx, ref, tol)
        if up:
            for name, got, v, ev, sv in (("dwg", self.dwg, dg, edg, sdg), ("dwu", self.dwu, du, edu, sdu)):
                self.near(name, got, x.t() @ v, x.t().abs() @ ev + self.M * E * (x.t().abs() @ sv), self.gt)
        if down:
            self.near("dwd", self.dwd, h.t() @ dy, self.M * E * (h.t().abs() @ dy.abs()), self.gt)
        self.untouched()

    def untouched(self):
        """The elements of the outputs' buffers outside the matrices."""
        for buf, v in self.bufs:
            rows, ld = (v.shape[0], v.stride(0)) if v.shape[1] <= 1 or v.stride(1) == 1 else (v.shape[1], v.stride(1))
            keep = self.t.ones_like(buf, dtype=self.t.bool)
            cols = ld - self.pad
            if rows and cols:
                keep[self.off:self.off + rows * ld].view(rows, ld)[:, :cols] = False
            assert (buf[keep] == 555.0).all()


# what the sizes run is asserted in test_sizes_cover_the_kernels
SIZES = [(1, 512, 1536), (5, 8, 16), (33, 264, 520), (64, 1024, 2048), (100, 72, 88), (300, 520, 1000), (520, 2048, 4096),
         (1000, 1000, 4096), (1300, 2048, 2816), (3000, 256, 256), (8200, 264, 512),
         (2048, 1024, 8192), (1777, 1000, 2728), (20, 1024, 8192), (60, 512, 8192),
         (16, 4096, 2048), (32, 1000, 1032), (17, 8200, 40), (1349, 1856, 6016), (785, 1408, 4800), (292, 1472, 5696), (3172, 2048, 2688)]
# sizes that are not whole chunks, misaligned pitches and addresses
ODD = [(1, 1, 1), (3, 7, 5), (17, 100, 77), (130, 333, 259), (257, 1001, 515), (1030, 515, 1033)]


def test_sizes_cover_the_kernels(t):
    fwd, bwd = set(), set()
    for s in SIZES + ODD:
        for layouts in (ac.AC_FFN_ROW, ac.AC_FFN_UP_COL):
            fwd |= {k.split(" x")[0] for k in ac.adaptcore_gated_ffn_kernels(*s, layouts=layouts)}
        bwd |= {k.split(" x")[0] for k in ac.adaptcore_gated_ffn_kernels(*s, backward=True)}
    assert {"k_gated<128, 128>", "k_gated<128, 128, 3>", "k_gated<128, 256>", "k_gated<256, 256>", "k_gated_sum", "k_multi<32, 128>", "k_rows<1>",
            "k_rows<2>"} <= fwd, fwd
    assert {"k_dgate<128, 128>", "k_dgate<128, 128, 3>", "k_dgate<256, 256>", "k_dgate_sum", "k_plain_sum",
            "k_multi<32, 128>", "k_multi<128, 128>", "k_multi<128, 128, 3>", "k_multi<128, 256>", "k_multi<256, 256>"} <= bwd, bwd


@pytest.mark.parametrize("layout", ["rr", "cc", "rc", "cr"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_block(t, size, layout):
    p = Problem(t, *size, layout=layout, dtype=t.float16 if layout in ("rc", "cr") else t.bfloat16)
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layout", ["rr", "cc"])
@pytest.mark.parametrize("size", ODD, ids=lambda s: "x".join(map(str, s)))
def test_odd_sizes(t, size, layout, dtype):
    p = Problem(t, *size, layout=layout, dtype=t.float16 if dtype == "f16" else t.bfloat16, pad=3, off=1)
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()


@pytest.mark.parametrize("pad,off", [(0, 1), (4, 0), (8, 0), (8, 8)])
def test_pitches(t, pad, off):
    """Sizes of whole chunks at addresses and pitches that are not, and that
    are."""
    p = Problem(t, 200, 256, 384, pad=pad, off=off)
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()


def test_one_misaligned_projection(t):
    p = Problem(t, 40, 128, 256, layout="cc")
    shifted = t.empty(256 * 128 + 1, dtype=p.dt, device="cuda")[1:].view(256, 128)
    shifted.copy_(p.wu.t())
    p.wu = shifted.t()
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh"])
@pytest.mark.parametrize("size", [(9, 64, 128), (600, 512, 2048)], ids=lambda s: "x".join(map(str, s)))
def test_activations(t, act, size):
    p = Problem(t, *size, act=act, dtype=t.float16)
    p.x.mul_(3.0)
    p.forward()
    p.check_forward()
    p.backward()
    p.check_backward()


@pytest.mark.parametrize("size", [(200, 256, 384), (5000, 128, 256), (77, 101, 203)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("layout", ["rr", "cc"])
def test_fp32_weight_gradients(t, size, layout):
    p = Problem(t, *size, layout=layout, grads=t.float32)
    p.forward()
    p.backward()
    p.check_backward()


def test_some_gradients_only(t):
    p = Problem(t, 300, 256, 512)
    p.forward()
    p.backward(dX=None)
    p.check_backward(dx=False)
    p.dx.fill_(0)
    p.backward(dWg=None, dWu=None, dWd=None)
    p.check_backward()
    p.dwd.fill_(0)
    p.backward(dX=None, dWg=None, dWu=None)
    p.check_backward()
    p.backward(dX=None, dWg=None, dWu=None, dWd=None)


def test_not_saved_and_first_half(t):
    for size in ((3, 256, 512), (700, 512, 2048)):
        p = Problem(t, *size)
        p.forward(save=False)
        p.check_forward(saved=False)
        assert (p.gate == 555.0).all() and (p.up == 555.0).all()
        h = p.h.clone()
        p.h.fill_(0)
        ac.gated_mm_tensors(p.x, p.wg, p.wu, p.h, gate=p.gate, up=p.up)
        assert t.equal(p.h, h)
        p.check_forward()


def test_empty(t):
    p = Problem(t, 0, 64, 32)
    p.forward()
    p.backward()
    assert not p.dwg.any() and not p.dwu.any() and not p.dwd.any()
    p = Problem(t, 5, 64, 0)
    p.forward()
    p.backward()
    assert not p.y.any() and not p.dx.any()
    p = Problem(t, 5, 0, 32)
    p.forward()
    p.backward()
    assert not p.h.any() and not p.gate.any()


def test_gradients_against_differences(t):
    """The pass as a whole: the loss sum(dy * y) along random directions of
    every input against the gradients, central differences in 64 bits of the
    formula; the gradients' own error is the roundings' (3 u of their norm)."""
    p = Problem(t, 60, 64, 96, dtype=t.float16)
    p.forward()
    p.backward()

    def loss(x, wg, wu, wd):
        a, _ = act64(t, p.act, x @ wg)
        return ((a * (x @ wu)) @ wd * p.dy.double()).sum()

    at = [v.double() for v in (p.x, p.wg, p.wu, p.wd)]
    for i, grad in enumerate((p.dx, p.dwg, p.dwu, p.dwd)):
        for _ in range(3):
            v = t.randn(at[i].shape, device="cuda", dtype=t.float64, generator=p.g)
            hi, lo = list(at), list(at)
            hi[i], lo[i] = at[i] + 1e-5 * v, at[i] - 1e-5 * v
            d = (loss(*hi) - loss(*lo)) / 2e-5
            # a direction of independent unit normals meets an error of norm n
            # with a value of standard deviation n
            assert abs((grad.double() * v).sum() - d) <= 5 * 3 * p.u * grad.double().norm() + 1e-6


def test_large_gates(t):
    """Gates far out on both sides: the activation saturates, nothing
    overflows on the way."""
    for act in ("silu", "gelu", "gelu_tanh"):
        p = Problem(t, 33, 64, 128, act=act)
        p.x.mul_(60.0)
        p.forward()
        p.check_forward()
        p.backward()
        p.check_backward()


def test_non_finite_rows_stay_alone(t):
    """A row with a NaN and one with an infinity leave the other rows' results
    as they were, also in tiles with padded K and in copies."""
    for size, pad in (((200, 72, 136), 0), ((130, 75, 139), 3)):
        p = Problem(t, *size, pad=pad)
        p.forward()
        clean = [v.clone() for v in (p.h, p.y)]
        p.backward()
        dx = p.dx.clone()
        p.x[3, 70], p.x[100, 0] = float("nan"), float("inf")
        p.dy[3, 1] = float("nan")
        p.forward()
        p.backward(dWg=None, dWu=None, dWd=None)
        rows = t.ones(size[0], dtype=t.bool, device="cuda")
        rows[3] = rows[100] = False
        for now, was in zip((p.h, p.y, p.dx), clean + [dx]):
            assert t.equal(now[rows], was[rows])
            assert t.isnan(now[3]).all()


def test_same_bits_and_other_stream(t):
    for size in ((7, 512, 1024), (900, 256, 1024)):
        outs = []
        for s in (t.cuda.current_stream(), t.cuda.Stream()):
            p = Problem(t, *size)
            t.cuda.synchronize()
            with t.cuda.stream(s):
                p.forward()
                p.backward()
            s.synchronize()
            outs.append([v.clone() for v in (p.h, p.y, p.dx, p.dwg, p.dwu, p.dwd)])
        for a, b in zip(*outs):
            assert t.equal(a, b)


def test_graph_replays(t):
    """Captured on a stream whose workspace is there, with copies, splits and
    sums in it; each replay on other inputs equals the eager call."""
    M, D, F = 70, 101, 333
    p = Problem(t, M, D, F)
    s = t.cuda.Stream()
    ac.adaptcore_reserve_workspace(s.cuda_stream, max(ac.adaptcore_gated_ffn_workspace(M, D, F),
                                                      ac.adaptcore_gated_ffn_workspace(M, D, F, backward=True)))
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph, stream=s):
        p.forward()
        p.backward()
    for i in range(4):
        p.x.copy_(t.randn(M, D, device="cuda"))
        t.cuda.synchronize()
        graph.replay()
        t.cuda.synchronize()
        outs = (p.h, p.y, p.dx, p.dwg, p.dwu, p.dwd)
        got = [v.clone() for v in outs]
        for v in outs:
            v.fill_(0)
        p.forward()
        p.backward()
        t.cuda.synchronize()
        for a, b in zip(got, outs):
            assert t.equal(a, b), i


def test_workspace_bounds_every_call(t):
    """The sizes the workspace function promises are enough: a call on a
    stream that has just that much, under capture, where nothing can grow."""
    for M, D, F in ((3, 129, 257), (500, 301, 203)):
        for layout in ("rr", "cc"):
            p = Problem(t, M, D, F, layout=layout, pad=1, off=1)
            s = t.cuda.Stream()
            ac.adaptcore_reserve_workspace(s.cuda_stream, max(ac.adaptcore_gated_ffn_workspace(M, D, F),
                                                              ac.adaptcore_gated_ffn_workspace(M, D, F, True)))
            t.cuda.synchronize()
            for kw in (dict(), dict(dWd=None), dict(dWg=None, dWu=None), dict(dX=None, dWg=None, dWu=None)):
                graph = t.cuda.CUDAGraph()
                with t.cuda.graph(graph, stream=s):
                    p.forward()
                    p.backward(**kw)


def test_refuses_tensors(t):
    p = Problem(t, 4, 16, 24)
    q = Problem(t, 4, 16, 24, layout="rr")
    ok = (p.x, p.wg, p.wu, p.wd, p.h, p.y)

    def sub(i, v):
        a = list(ok)
        a[i] = v
        return a

    for a in (sub(0, p.x.float()), sub(1, p.wg.float()), sub(2, p.wu.half()), sub(3, p.wd.half()), sub(4, p.h.float()),
              sub(5, p.y.float())):
        with pytest.raises(TypeError):
            ac.gated_ffn_tensors(*a)
    for a in (sub(2, q.wu), sub(1, p.wg[:, :20]), sub(3, p.wd.t()), sub(4, p.h[:3]), sub(5, p.y.cpu()),
              sub(1, p.wg[::2])):
        with pytest.raises(ValueError):
            ac.gated_ffn_tensors(*a)
    with pytest.raises(ValueError):
        ac.gated_ffn_tensors(*ok, act="relu")
    with pytest.raises(ValueError):
        ac.gated_ffn_tensors(*ok, gate=p.gate)
    with pytest.raises(ValueError):
        p.backward(dWg=None)
    with pytest.raises(ValueError):
        p.backward(dWg=q.dwg, dWu=q.dwu)
    with pytest.raises(ValueError):
        p.backward(dWd=q.dwd)
    with pytest.raises(TypeError):
        p.backward(dWd=t.empty(16, 24, device="cuda").t())


def test_backward_after_a_block_of_twice_the_features(t):
    """(the second product of the one and dX of the other differ in their
    k-blocks alone)"""
    for M, D, F in ((128, 128, 96), (300, 72, 32)):
        p = Problem(t, M, D, 2 * F)
        p.forward()
        p.check_forward()
        p = Problem(t, M, D, F)
        p.forward()
        p.backward()
        p.check_backward()


def test_one_row_of_any_stride(t):
    """A single token is one row, however far the next one would lie: the last
    position of a long sequence, columns of a wide buffer."""
    far = 2 ** 23 + 64

    def one(n, fill=None):
        v = t.empty(1, far, device="cuda", dtype=t.bfloat16)[:, 64:64 + n]
        return v.copy_(fill) if fill is not None else v

    p = Problem(t, 1, 256, 384)
    p.forward()
    p.backward()
    x, dy, h, y, gate, up, dx = (one(n) for n in (256, 256, 384, 256, 384, 384, 256))
    x.copy_(p.x), dy.copy_(p.dy)
    gate = t.empty(1, 1000, device="cuda", dtype=t.bfloat16)[:, :384]  # (another stride than up's)
    ac.gated_ffn_tensors(x, p.wg, p.wu, p.wd, h, y, gate=gate, up=up)
    assert t.equal(h, p.h) and t.equal(y, p.y) and t.equal(gate, p.gate) and t.equal(up, p.up)
    ac.gated_mm_tensors(x, p.wg, p.wu, h.zero_())
    assert t.equal(h, p.h)
    dwg, dwu, dwd = t.empty_like(p.dwg), t.empty_like(p.dwu), t.empty_like(p.dwd)
    ac.gated_ffn_backward_tensors(dy, x, p.wg, p.wu, p.wd, gate, up, h, dX=dx, dWg=dwg, dWu=dwu, dWd=dwd)
    assert t.equal(dx, p.dx) and t.equal(dwg, p.dwg) and t.equal(dwu, p.dwu) and t.equal(dwd, p.dwd)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("size", [(33, 64, 128), (300, 520, 1000)], ids=lambda s: "x".join(map(str, s)))
def test_saved_gates_whose_square_overflows(t, act, size):
    """The activation's derivative is 0 or 1 far out, not 0 * infinity."""
    p = Problem(t, *size, act=act)
    p.forward()
    p.gate.fill_(1e20)
    p.gate[:, ::3] = -1e20
    p.gate[:, 1::5] = -3e19
    p.backward()
    p.check_backward()
