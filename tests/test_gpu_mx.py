"""The microscaled 4-bit operators on the GPU against the 64-bit forms.

Codes, scales and values have to be equal. A product's terms are exact in fp32
(two bits times two bits times a power of two), and so is a sum's error at most
e = 2^-24 (half a unit) times the sum of the terms' magnitudes for every addition
of a partial sum: the instructions' own (one for 32 terms at least: K / 32), and 64
for the waves and partitions whose sums are added. The result's rounding adds u |y|,
u = 2^-8 (bf16), 2^-11 (fp16, and 2^-25 where it is subnormal), e.
"""
import numpy as np
import pytest

import paper_2608_10803_amd as ac
from oracle import mx_ref

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
    return x.detach().double().cpu().numpy()


def view(t, rows, cols, dtype, pad=0, off=0, canary=77):
    """rows x cols view of a larger canary buffer, and the buffer."""
    buf = t.full(((rows + 1) * (cols + pad) + off,), canary, dtype=dtype, device="cuda")
    return buf[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols], buf


def untouched(t, v, buf, canary=77):
    """The buffer around the view still holds the canary."""
    v.fill_(canary)
    return bool((buf == canary).all())


def operand(t, r, rows, cols, spread=6, pad=0, off=0):
    """Random codes and scales of a rows x cols matrix on the GPU (zeros past
    cols, scales of 2 spread + 1 powers of two), and its 64-bit values."""
    cs, ss = mx_ref.shapes(rows, cols)
    codes = r.integers(0, 256, size=cs).astype(np.uint8)
    if cols % 32:
        k = cols % 32
        tail = codes[:, -16:]
        tail[:, (k + 1) // 2:] = 0
        if k % 2:
            tail[:, k // 2] &= 15
    scales = r.integers(127 - spread, 127 + spread + 1, size=ss).astype(np.uint8)
    dc, _ = view(t, *cs, t.uint8, pad, off)
    ds, _ = view(t, *ss, t.uint8, pad, off)
    dc.copy_(t.from_numpy(codes))
    ds.copy_(t.from_numpy(scales))
    return dc, ds, mx_ref.values(codes, scales, cols)


def inputs(r, rows, cols, dtype):
    """Values with whole blocks of zeros, of subnormal and of the largest
    magnitudes, ties, and (rows from 3 on) infinities and NaN."""
    x = r.normal(size=(rows, cols)) * np.exp2(r.integers(-6, 6, size=(rows, cols)).astype(float))
    pick = r.random((rows, cols)) < 0.3
    x = np.where(pick, r.choice([0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, -0.25, -5, -0.0], size=(rows, cols)), x)
    n = -(-cols // 32)
    for i in range(rows):
        b = slice(32 * int(r.integers(n)), None)
        b = slice(b.start, min(b.start + 32, cols))
        kind = i % 7
        if kind == 1:
            x[i, b] = 0
        elif kind == 2:
            x[i, b] *= {"f32": 2.0 ** -140, "bf16": 2.0 ** -132, "f16": 2.0 ** -20}[dtype]
        elif kind == 3:
            x[i, b.start] = [np.inf, -np.inf, np.nan][i % 3]
        elif kind == 4:
            x[i, b.start] = {"f32": 3.4e38, "bf16": 3.3e38, "f16": 65504.0}[dtype]
    return x


SIZES = [(1, 1), (3, 7), (8, 32), (9, 33), (2, 511), (33, 512), (600, 1000), (65, 1531), (17, 5000), (257, 4096), (130, 259),
         (1, 4096), (4096, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "%dx%d" % s)
def test_quantize(t, size, dtype):
    rows, cols = size
    r = np.random.default_rng(rows * 7 + cols)
    x = t.from_numpy(inputs(r, rows, cols, dtype)).to("cuda").to(dt(t, dtype))
    codes, scales = mx_ref.quantize(f64(x))
    cs, ss = ac.mxfp4_shapes(rows, cols)
    for layout in "rc":
        for pad, off in ((0, 0), (5, 3)):
            if layout == "r":
                xv, _ = view(t, rows, cols, x.dtype, pad, off)
                xv.copy_(x)
            else:
                xv, _ = view(t, cols, rows, x.dtype, pad, off)
                xv.copy_(x.t())
                xv = xv.t()
            c, cbuf = view(t, *cs, t.uint8, pad, off)
            s, sbuf = view(t, *ss, t.uint8, pad, off)
            ac.mxfp4_quantize_tensors(xv, c, s)
            assert np.array_equal(s.cpu().numpy(), scales), (layout, pad)
            assert np.array_equal(c.cpu().numpy(), codes), (layout, pad)
            want = mx_ref.values(codes, scales, cols)
            for out in ("f32", "bf16", "f16"):
                y, ybuf = view(t, rows, cols, dt(t, out), pad, off)
                ac.mxfp4_dequantize_tensors(c, s, y)
                ref = t.from_numpy(want).to("cuda").to(t.float32).to(dt(t, out))
                assert t.equal(t.nan_to_num(y.float(), nan=123.0), t.nan_to_num(ref.float(), nan=123.0)), out
                assert t.equal(t.signbit(y) | t.isnan(y), t.signbit(ref) | t.isnan(ref)), out
                assert untouched(t, y, ybuf)
            assert untouched(t, c, cbuf) and untouched(t, s, sbuf)


def test_every_code_and_scale(t):
    """All 16 codes under all 256 scales."""
    codes = t.arange(16, dtype=t.uint8).view(1, 8, 2)
    codes = (codes[:, :, 0] + 16 * codes[:, :, 1]).repeat(256, 2).contiguous().cuda()
    scales = t.arange(256, dtype=t.uint8).view(256, 1).contiguous().cuda()
    y = t.empty(256, 32, device="cuda")
    ac.mxfp4_dequantize_tensors(codes, scales, y)
    want = mx_ref.values(codes.cpu().numpy(), scales.cpu().numpy(), 32)
    got = f64(y)
    # (from 2 x 2^127 on past the largest fp32 value, (2 - 2^-23) 2^127)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    assert np.array_equal(np.nan_to_num(got, nan=1.5, posinf=9e300, neginf=-9e300),
                          np.nan_to_num(want, nan=1.5, posinf=9e300, neginf=-9e300))


def check(got, ref, mag, K, out, extra=0.0):
    tol = (K / 32 + 64) * E * mag + extra
    tol = tol + UNIT[out] * (np.abs(ref) + tol) + TINY[out]
    bad = np.abs(got - ref) > tol
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])


PRODUCTS = [(1, 1, 1), (1, 16, 32), (2, 17, 33), (3, 100, 511), (15, 64, 128), (16, 70, 4096), (17, 33, 1000), (31, 48, 96),
            (33, 130, 160), (64, 256, 513), (65, 257, 255), (127, 129, 1024), (128, 256, 2048), (129, 300, 1001), (200, 511, 64),
            (300, 640, 300), (1, 4096, 14336), (5, 2000, 7000), (257, 513, 4096), (520, 1031, 769)]


@pytest.mark.parametrize("size", PRODUCTS, ids=lambda s: "%dx%dx%d" % s)
def test_product(t, size):
    M, N, K = size
    r = np.random.default_rng(M * 11 + N + K)
    for out, pad, off in (("bf16", 0, 0), ("f32", 3, 1), ("f16", 16, 16)):
        a, sa, A = operand(t, r, M, K, pad=pad, off=off)
        b, sb, B = operand(t, r, N, K, pad=pad, off=off)
        scale = 2.0 ** -10 if out == "f16" else 1.0  # (inside fp16's range)
        if out == "f16":
            sb -= 10
            B = B * scale
        bias = t.from_numpy(r.normal(size=N)).float().cuda() if pad else None
        y, ybuf = view(t, M, N, dt(t, out), pad, off)
        ac.mxfp4_mm_tensors(a, b, sb, y, A_scales=sa, bias=bias)
        mag = np.abs(A) @ np.abs(B).T
        ref = mx_ref.product(A, B)
        if bias is not None:
            ref, mag = ref + f64(bias), mag + np.abs(f64(bias))
        check(f64(y), ref, mag, K, out)
        assert untouched(t, y, ybuf)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", [(1, 70, 1), (1, 300, 4096), (4, 33, 77), (16, 64, 4096), (33, 100, 1001), (130, 257, 515),
                                  (300, 256, 1024)], ids=lambda s: "%dx%dx%d" % s)
def test_product_quantises_its_left_operand(t, size, dtype):
    """16-bit and 32-bit values: the bits of the call on their codes."""
    M, N, K = size
    r = np.random.default_rng(M + N + K)
    x, _ = view(t, M, K, dt(t, dtype), 3, 1)
    x.copy_(t.from_numpy(r.normal(size=(M, K))))
    b, sb, B = operand(t, r, N, K)
    y = t.empty(M, N, device="cuda")
    ac.mxfp4_mm_tensors(x, b, sb, y)
    X = mx_ref.rounded(f64(x))
    check(f64(y), mx_ref.product(X, B), np.abs(X) @ np.abs(B).T, K, "f32")


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("size", [(1, 1, 1), (1, 64, 256), (3, 33, 100), (16, 200, 2048), (17, 100, 1001), (40, 129, 512),
                                  (64, 128, 96), (129, 130, 515), (260, 300, 1024), (513, 257, 160)],
                         ids=lambda s: "%dx%dx%d" % s)
def test_gated(t, size, act):
    M, F, K = size
    r = np.random.default_rng(M + F + K)
    for out, a4 in (("bf16", True), ("f16", False), ("f32", True)):
        # gates of about unit size
        unit = int(np.round(np.log2(9.0 * np.sqrt(K))))
        bg, sg, G = operand(t, r, F, K, spread=1)
        bu, su, U = operand(t, r, F, K, spread=1)
        sg -= unit
        su -= unit
        G, U = G * 2.0 ** -unit, U * 2.0 ** -unit
        h, hbuf = view(t, M, F, dt(t, out), 3, 1)
        if a4:
            a, sa, A = operand(t, r, M, K, spread=1)
            ac.mxfp4_gated_mm_tensors(a, bg, sg, bu, su, h, A_scales=sa, act=act)
        else:
            x = t.from_numpy(2.0 * r.normal(size=(M, K))).cuda().to(dt(t, out))
            A = mx_ref.rounded(f64(x))
            ac.mxfp4_gated_mm_tensors(x, bg, sg, bu, su, h, act=act)
        ref, g, u = mx_ref.gated(A, G, U, act)
        eg = (K / 32 + 64) * E * (np.abs(A) @ np.abs(G).T)
        eu = (K / 32 + 64) * E * (np.abs(A) @ np.abs(U).T)
        # the activation: a slope of at most 1.13, its own arithmetic (an exponential and a
        # reciprocal to some units, and the exponent's rounding: |g| units)
        a = np.abs(mx_ref.activation(act, g)[0])
        tol = 1.13 * eg * (np.abs(u) + eu) + a * eu + 16 * E * (1 + np.abs(g)) * (a + 1e-30) * (np.abs(u) + eu)
        if act == "gelu":  # 1 + erf loses the digits that a value close to -1 takes
            tol = tol + 8 * E * np.abs(g) * np.abs(u)
        tol = tol + UNIT[out] * (np.abs(ref) + tol) + TINY[out]
        assert (np.abs(f64(h) - ref) <= tol).all(), (out, np.max(np.abs(f64(h) - ref) / tol))
        assert untouched(t, h, hbuf)


# sizes whose products run on each of the tiles, whole and split along K
TILES = [("k_mx_tile<32, 128>", 523, 77, 300), ("k_mx_tile<32, 128> x24", 41, 71, 30000),
         ("k_mx_tile<32, 128> x3", 520, 512, 8192), ("k_mx_tile<128, 128>", 130, 8199, 64),
         ("k_mx_tile<128, 128> x8", 4096, 64, 30000), ("k_mx_tile<64, 256>", 520, 4096, 4096),
         ("k_mx_tile<64, 256> x4", 131, 4095, 14336), ("k_mx_tile<128, 256>", 523, 8192, 4096),
         ("k_mx_tile<128, 256> x4", 130, 8192, 30000), ("k_mx_tile<256, 256>", 2047, 8191, 4100),
         ("k_mx_tile<256, 256> x3", 1100, 4096, 30000)]
GATED_TILES = [("k_mx_tile<128, 128>", 523, 71, 100), ("k_mx_tile<128, 128> x8", 520, 64, 4096),
               ("k_mx_tile<64, 256>", 520, 67, 2048), ("k_mx_tile<64, 256> x12", 33, 65, 14336),
               ("k_mx_tile<128, 256>", 520, 4096, 4096), ("k_mx_tile<128, 256> x4", 130, 4096, 30000),
               ("k_mx_tile<256, 256>", 1024, 8192, 4096), ("k_mx_tile<256, 256> x3", 1100, 2048, 30000)]


def random_operand(t, g, rows, cols, spread):
    """An operand as `operand` makes them, by the GPU, and its values in 64 bits by
    elementary operations."""
    cs, ss = ac.mxfp4_shapes(rows, cols)
    codes = t.randint(0, 256, cs, generator=g, device="cuda", dtype=t.uint8)
    if cols % 32:
        k = cols % 32
        codes[:, cs[1] - 16 + (k + 1) // 2:] = 0
        if k % 2:
            codes[:, cs[1] - 16 + k // 2] &= 15
    scales = t.randint(127 - spread, 128 + spread, ss, generator=g, device="cuda", dtype=t.uint8)
    c = t.stack((codes & 15, codes >> 4), 2).view(rows, -1).long()
    lut = t.tensor(np.concatenate((mx_ref.LEVELS, -mx_ref.LEVELS)), device="cuda")
    unit = t.pow(t.tensor(2.0, dtype=t.float64, device="cuda"), scales.double() - 127.0)
    return codes, scales, (lut[c].view(rows, -1, 32) * unit[:, :, None]).view(rows, -1)[:, :cols].contiguous()


def same_on_gpu(t, got, ref, mag, K, out, extra=0.0):
    tol = (K / 32 + 64) * E * mag + extra
    tol = tol + UNIT[out] * (ref.abs() + tol) + TINY[out]
    worst = float(((got.double() - ref).abs() / tol).max())
    assert worst <= 1.0, worst


@pytest.mark.parametrize("kernel,M,N,K", TILES, ids=lambda v: str(v))
def test_every_tile(t, kernel, M, N, K):
    assert ac.adaptcore_mxfp4_kernels(M, N, K)[1] == kernel
    g = t.Generator(device="cuda").manual_seed(M + N + K)
    a, sa, A = random_operand(t, g, M, K, 4)
    b, sb, B = random_operand(t, g, N, K, 4)
    ref, mag = A @ B.t(), A.abs() @ B.abs().t()
    del A, B
    bias = t.randn(N, device="cuda", generator=g) * 100
    for out in ("bf16", "f32", "f16"):
        scale = 2.0 ** -12 if out == "f16" else 1.0  # (inside fp16's range)
        if out == "f16":
            sb -= 12
        y, ybuf = view(t, M, N, dt(t, out), 5, 3)
        ac.mxfp4_mm_tensors(a, b, sb, y, A_scales=sa)
        same_on_gpu(t, y, ref * scale, mag * scale, K, out)
        z = t.empty(M, N, device="cuda", dtype=dt(t, out))
        ac.mxfp4_mm_tensors(a, b, sb, z, A_scales=sa, bias=bias)
        same_on_gpu(t, z, ref * scale + bias.double(), mag * scale + bias.double().abs(), K, out)
        assert untouched(t, y, ybuf)


@pytest.mark.parametrize("kernel,M,F,K", GATED_TILES, ids=lambda v: str(v))
def test_every_gated_tile(t, kernel, M, F, K):
    assert ac.adaptcore_mxfp4_kernels(M, F, K, True)[1] == kernel
    g = t.Generator(device="cuda").manual_seed(M + F + K)
    a, sa, A = random_operand(t, g, M, K, 1)
    bg, sg, G = random_operand(t, g, F, K, 1)
    bu, su, U = random_operand(t, g, F, K, 1)
    unit = int(np.round(np.log2(9.0 * np.sqrt(K))))
    sg -= unit
    su -= unit
    G, U = G * 2.0 ** -unit, U * 2.0 ** -unit
    gate, up = A @ G.t(), A @ U.t()
    eg, eu = ((K / 32 + 64) * E * (A.abs() @ w.abs().t()) for w in (G, U))
    del A, G, U
    for act in ("silu", "gelu", "gelu_tanh"):
        fn = {"silu": t.nn.functional.silu, "gelu": t.nn.functional.gelu,
              "gelu_tanh": lambda x: t.nn.functional.gelu(x, approximate="tanh")}[act]
        value = fn(gate)
        for out in ("bf16", "f32", "f16"):
            h, hbuf = view(t, M, F, dt(t, out), 5, 3)
            ac.mxfp4_gated_mm_tensors(a, bg, sg, bu, su, h, A_scales=sa, act=act)
            # (the terms of test_gated)
            v = value.abs()
            tol = 1.13 * eg * (up.abs() + eu) + v * eu + 16 * E * (1 + gate.abs()) * (v + 1e-30) * (up.abs() + eu)
            if act == "gelu":
                tol = tol + 8 * E * gate.abs() * up.abs()
            ref = value * up
            tol = tol + UNIT[out] * (ref.abs() + tol) + TINY[out]
            worst = float(((h.double() - ref).abs() / tol).max())
            assert worst <= 1.0, (act, out, worst)
            assert untouched(t, h, hbuf)


@pytest.mark.parametrize("size", [(1, 300, 500), (16, 4096, 1000), (20, 130, 3001), (40, 600, 2049), (300, 600, 1100)],
                         ids=lambda s: "%dx%dx%d" % s)
def test_alignments_give_the_same_bits(t, size):
    """Operands at any pitch and address: the bits of aligned ones (the same kernel
    but for its loads, or copies first)."""
    M, N, K = size
    g = t.Generator(device="cuda").manual_seed(M)
    a, sa, _ = random_operand(t, g, M, K, 3)
    b, sb, _ = random_operand(t, g, N, K, 3)
    b2, sb2, _ = random_operand(t, g, N, K, 3)

    def run(*ops):
        y, h = t.empty(M, N, device="cuda"), t.empty(M, N, device="cuda")
        ac.mxfp4_mm_tensors(ops[0], ops[2], ops[3], y, A_scales=ops[1])
        ac.mxfp4_gated_mm_tensors(ops[0], ops[2], ops[3], ops[4], ops[5], h, A_scales=ops[1])
        return y, h

    def moved(x, pad, off):
        v, _ = view(t, *x.shape, t.uint8, pad, off, 255)
        v.copy_(x)
        return v

    same = ac.adaptcore_mxfp4_kernels(M, N, K) and M <= 32  # (other sizes may run on other kernels misaligned)
    want = run(a, sa, b, sb, b2, sb2)
    for pa, pb in (((0, 0), (7, 5)), ((7, 5), (0, 0)), ((1, 1), (3, 2)), ((16, 16), (48, 32))):
        got = run(moved(a, *pa), moved(sa, *pa), moved(b, *pb), moved(sb, *pb), moved(b2, *pb), moved(sb2, *pb))
        for x, y in zip(got, want):
            if same:
                assert t.equal(x, y), (pa, pb)
            else:  # sums in another order: both within K / 32 + 64 units of the terms' magnitudes
                assert float((x - y).abs().max()) <= 2 * (K / 32 + 64) * E * float(y.abs().max()) * 40, (pa, pb)


@pytest.mark.parametrize("size", [(1, 300, 500), (20, 130, 3001), (40, 600, 2049), (130, 257, 515), (300, 600, 1100),
                                  (700, 130, 4000)], ids=lambda s: "%dx%dx%d" % s)
def test_every_element_at_any_alignment(t, size):
    """Operands at any pitch and address, on rows or tiles, whichever a call then
    chooses: every element against the 64-bit form."""
    M, N, K = size
    g = t.Generator(device="cuda").manual_seed(M + N)
    a, sa, A = random_operand(t, g, M, K, 3)
    b, sb, B = random_operand(t, g, N, K, 3)
    b2, sb2, B2 = random_operand(t, g, N, K, 3)
    gate, up = A @ B.t(), A @ B2.t()
    mag = [A.abs() @ m.abs().t() for m in (B, B2)]
    e = [(K / 32 + 64) * E * m for m in mag]
    ref = gate * t.sigmoid(gate) * up
    # (the terms of test_gated)
    tol = 1.13 * e[0] * (up.abs() + e[1]) + gate.abs() * e[1] + 16 * E * (1 + gate.abs()) * (gate.abs() + 1e-30) * (up.abs() + e[1])
    tol = tol + E * (ref.abs() + tol)

    def moved(x, pad, off):
        v, _ = view(t, *x.shape, t.uint8, pad, off, 255)
        v.copy_(x)
        return v

    for pa, pb in (((0, 0), (0, 0)), ((0, 0), (7, 5)), ((7, 5), (0, 0)), ((1, 1), (3, 2)), ((16, 16), (48, 32)), ((16, 3), (16, 7))):
        ops = [moved(v, *p) for v, p in ((a, pa), (sa, pa), (b, pb), (sb, pb), (b2, pb), (sb2, pb))]
        y, ybuf = view(t, M, N, t.float32, *pa)
        h, hbuf = view(t, M, N, t.float32, *pb)
        ac.mxfp4_mm_tensors(ops[0], ops[2], ops[3], y, A_scales=ops[1])
        ac.mxfp4_gated_mm_tensors(ops[0], ops[2], ops[3], ops[4], ops[5], h, A_scales=ops[1])
        same_on_gpu(t, y, gate, mag[0], K, "f32")
        assert float(((h.double() - ref).abs() / tol).max()) <= 1.0, (pa, pb)
        assert untouched(t, y, ybuf) and untouched(t, h, hbuf)


def test_empty_depth(t):
    e = t.empty(5, 0, device="cuda", dtype=t.uint8)
    y, bias = t.full((5, 5), 7.0, device="cuda"), t.arange(5, device="cuda", dtype=t.float32)
    ac.mxfp4_mm_tensors(e, e, e, y, A_scales=e, bias=bias)
    assert t.equal(y, bias.expand(5, 5))
    ac.mxfp4_gated_mm_tensors(e, e, e, e, e, y, A_scales=e)
    assert not y.any()


def test_nan_blocks_stay_in_their_rows(t):
    r = np.random.default_rng(1)
    for M, N, K in ((5, 40, 256), (140, 300, 1024)):
        a, sa, A = operand(t, r, M, K)
        b, sb, B = operand(t, r, N, K)
        clean = t.empty(M, N, device="cuda")
        ac.mxfp4_mm_tensors(a, b, sb, clean, A_scales=sa)
        sa[3, 2] = 255
        sb[7, 1] = 255
        y = t.empty(M, N, device="cuda")
        ac.mxfp4_mm_tensors(a, b, sb, y, A_scales=sa)
        assert t.isnan(y[3]).all() and t.isnan(y[:, 7]).all()
        keep = t.ones(M, N, dtype=t.bool, device="cuda")
        keep[3], keep[:, 7] = False, False
        assert t.equal(y[keep], clean[keep])


def test_what_lies_beside_an_operand_does_not_count(t):
    """Pitches with NaN scales and full codes in the padding."""
    r = np.random.default_rng(2)
    for M, N, K in ((4, 50, 200), (150, 260, 200), (150, 260, 1056)):
        got = []
        for pad in (0, 16):
            r2 = np.random.default_rng(7)
            ops = []
            for rows in (M, N):
                c, s, _ = operand(t, r2, rows, K)
                cv, cbuf = view(t, *c.shape, t.uint8, pad, 0, 255)
                sv, sbuf = view(t, *s.shape, t.uint8, pad, 0, 255)
                cv.copy_(c)
                sv.copy_(s)
                ops.append((cv, sv))
            y = t.empty(M, N, device="cuda")
            ac.mxfp4_mm_tensors(ops[0][0], ops[1][0], ops[1][1], y, A_scales=ops[0][1])
            got.append(y)
        assert t.equal(got[0], got[1]), (M, N, K)


def test_other_stream_same_bits(t):
    r = np.random.default_rng(4)
    x = t.from_numpy(r.normal(size=(300, 1000))).cuda().bfloat16()
    b, sb, _ = operand(t, r, 500, 1000)

    def both(stream):
        y = t.empty(300, 500, device="cuda")
        with t.cuda.stream(stream):
            ac.mxfp4_mm_tensors(x, b, sb, y)
        stream.synchronize()
        return y

    t.cuda.synchronize()
    assert t.equal(both(t.cuda.current_stream()), both(t.cuda.Stream()))


def test_graph_replays(t):
    """Captured products, with eager work between the replays, equal the eager
    results every time."""
    r = np.random.default_rng(6)
    for M, N, K in ((3, 700, 2000), (200, 512, 3000)):
        x = t.from_numpy(r.normal(size=(M, K))).cuda().bfloat16()
        b, sb, _ = operand(t, r, N, K)
        b2, sb2, _ = operand(t, r, N, K)
        sb -= 8
        sb2 -= 8
        y, h = t.empty(M, N, device="cuda"), t.empty(M, N, device="cuda", dtype=t.bfloat16)

        def call():
            ac.mxfp4_mm_tensors(x, b, sb, y)
            ac.mxfp4_gated_mm_tensors(x, b, sb, b2, sb2, h)

        s = t.cuda.Stream()
        with t.cuda.stream(s):
            ac.adaptcore_reserve_workspace(s.cuda_stream, max(ac.adaptcore_mxfp4_workspace(M, N, K, g) for g in (0, 1)))
        t.cuda.synchronize()
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph, stream=s):
            call()
        for i in range(4):
            x.copy_(t.from_numpy(r.normal(size=(M, K))))
            t.cuda.synchronize()
            graph.replay()
            t.cuda.synchronize()
            got = y.clone(), h.clone()
            call()
            t.cuda.synchronize()
            assert t.equal(got[0], y) and t.equal(got[1], h), i


@pytest.mark.parametrize("size", [(5, 300, 1000), (40, 600, 2049), (300, 600, 1100), (64, 4096, 4096)],
                         ids=lambda s: "%dx%dx%d" % s)
@pytest.mark.parametrize("values", [False, True])
def test_captured_at_any_alignment(t, size, values):
    """What adaptcore_mxfp4_workspace says is enough wherever the operands lie, one
    of a pair alone at an odd address too."""
    M, N, K = size
    r = np.random.default_rng(M)
    x = t.from_numpy(r.normal(size=(M, K))).cuda().bfloat16()
    ops = [operand(t, r, rows, K)[:2] for rows in (M, N, N)]
    bias = t.from_numpy(r.normal(size=N)).float().cuda()
    y, h = t.empty(M, N, device="cuda"), t.empty(M, N, device="cuda")

    def moved(v, pad, off):
        to, _ = view(t, *v.shape, t.uint8, pad, off, 255)
        to.copy_(v)
        return to

    def call(a, sa, b, sb, b2, sb2):
        a, sa = (x, None) if values else (a, sa)
        ac.mxfp4_mm_tensors(a, b, sb, y, A_scales=sa, bias=bias)
        ac.mxfp4_gated_mm_tensors(a, b, sb, b2, sb2, h, A_scales=sa)

    call(*(v for pair in ops for v in pair))
    want = y.clone(), h.clone()
    A, B, B2 = (mx_ref.values(c.cpu().numpy(), s.cpu().numpy(), K) for c, s in ops)
    A = mx_ref.rounded(f64(x)) if values else A
    dot = [np.abs(A) @ np.abs(b).T for b in (B, B2)]
    _, gate, up = mx_ref.gated(A, B, B2, "silu")
    tol = [(K / 32 + 66) * E * (dot[0] + np.abs(f64(bias))),
           (K / 32 + 66) * E * (1.1 * dot[0] * np.abs(up) + np.abs(gate) * dot[1]) + 16 * E * np.abs(gate * up)]
    for offs in ((0, 0, 0), (1, 0, 0), (0, 3, 3), (5, 1, 7), (0, 0, 1), (2, 1, 0)):
        moves = [moved(v, 16, o) for (pair, o) in zip(ops, offs) for v in pair]
        s = t.cuda.Stream()
        ac.adaptcore_reserve_workspace(s.cuda_stream, max(ac.adaptcore_mxfp4_workspace(M, N, K, g) for g in (0, 1)))
        t.cuda.synchronize()
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph, stream=s):
            call(*moves)
        for _ in range(2):
            y.fill_(7)
            h.fill_(7)
            t.cuda.synchronize()
            graph.replay()
            t.cuda.synchronize()
            for got, ref, e in zip((y, h), want, tol):  # (sums in two orders, each within the half of it)
                assert (np.abs(f64(got) - f64(ref)) <= 2 * e).all(), offs


@pytest.mark.parametrize("stages", [1, 3, 9, 20, 34])
@pytest.mark.parametrize("M", [1, 16, 20])
@pytest.mark.parametrize("N", [70, 4130])
def test_few_rows_of_any_depth(t, M, N, stages):
    """The kernels of few rows with one stage of 512 k a wave, with several, and with
    waves that have one less, in all their forms: A in codes or in values, B aligned or
    not, plain and gated."""
    K = 512 * stages - 37
    g = t.Generator(device="cuda").manual_seed(M + N + K)
    x = t.randn(M, K, device="cuda", generator=g).bfloat16()
    cs, ss = ac.mxfp4_shapes(M, K)
    a, sa = t.empty(cs, dtype=t.uint8, device="cuda"), t.empty(ss, dtype=t.uint8, device="cuda")
    ac.mxfp4_quantize_tensors(x, a, sa)
    X = t.from_numpy(mx_ref.rounded(f64(x))).cuda()
    b, sb, B = random_operand(t, g, N, K, 3)
    b2, sb2, B2 = random_operand(t, g, N, K, 3)
    odd = []
    for v in (b, b2):
        odd.append(view(t, *v.shape, t.uint8, 3, 1, 255)[0])
        odd[-1].copy_(v)
    y, h = t.empty(M, N, device="cuda"), t.empty(M, N, device="cuda")
    gate, up = X @ B.t(), X @ B2.t()
    e = [(K / 32 + 64) * E * (X.abs() @ m.abs().t()) for m in (B, B2)]
    del B, B2
    ref = gate * t.sigmoid(gate) * up
    tol = 1.1 * e[0] * (up.abs() + e[1]) + gate.abs() * e[1] + 16 * E * (1 + gate.abs()) * ref.abs()
    for c, c2 in ((b, b2), odd):
        for left in ((x, None), (a, sa)):
            y.fill_(7)
            h.fill_(7)
            ac.mxfp4_mm_tensors(left[0], c, sb, y, A_scales=left[1])
            ac.mxfp4_gated_mm_tensors(left[0], c, sb, c2, sb2, h, A_scales=left[1])
            assert bool(((y.double() - gate).abs() <= e[0] + E * gate.abs()).all())
            assert bool(((h.double() - ref).abs() <= tol + E * ref.abs()).all())


@pytest.mark.parametrize("size", [(1, 300, 512), (3, 70, 1000), (16, 64, 700)], ids=lambda s: "%dx%dx%d" % s)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_values_beside_codes_at_odd_addresses(t, size, dtype):
    """The left operand quantised by the product's own kernel, where the codes of
    the right one are not loaded into LDS."""
    M, N, K = size
    r = np.random.default_rng(M + K)
    x = t.from_numpy(r.normal(size=(M, K))).cuda().to(dt(t, dtype))
    X = mx_ref.rounded(f64(x))
    ops = []
    for pad, off in ((0, 0), (5, 3)):
        r2 = np.random.default_rng(9)
        b, sb, B = operand(t, r2, N, K, pad=pad, off=off)
        b2, sb2, B2 = operand(t, r2, N, K, pad=pad, off=off)
        y, h = t.empty(M, N, device="cuda"), t.empty(M, N, device="cuda")
        ac.mxfp4_mm_tensors(x, b, sb, y)
        ac.mxfp4_gated_mm_tensors(x, b, sb, b2, sb2, h)
        ops.append((y, h))
    check(f64(ops[0][0]), mx_ref.product(X, B), np.abs(X) @ np.abs(B).T, K, "f32")
    check(f64(ops[1][0]), mx_ref.product(X, B), np.abs(X) @ np.abs(B).T, K, "f32")
    ref, gate, up = mx_ref.gated(X, B, B2, "silu")
    e = (K / 32 + 64) * E * (1.1 * (np.abs(X) @ np.abs(B).T) * np.abs(up) + np.abs(gate) * (np.abs(X) @ np.abs(B2).T))
    for y, h in ops:
        assert (np.abs(f64(h) - ref) <= e + 16 * E * np.abs(gate * up)).all()


@pytest.mark.parametrize("M", [3, 20, 150])
def test_scales_of_all_sizes(t, M):
    """Every scale byte but NaN's, in products that stay in fp32's range, and in
    some that leave it. (A partial sum below 2^-126 may be taken for zero: each of
    the K / 32 + 64 additions may lose that.)"""
    N, K = 260, 320
    r = np.random.default_rng(M)
    a, sa, _ = operand(t, r, M, K)
    b, sb, _ = operand(t, r, N, K)
    blocks = sa.shape[1]
    for total in (254, 140, 330, 100):
        p = t.from_numpy(r.integers(max(0, total - 254), min(254, total) + 1, size=blocks).astype(np.uint8)).cuda()
        p[0], p[1] = max(0, total - 254), min(254, total)
        sa[:] = p
        sb[:] = total - p
        y = t.empty(M, N, device="cuda")
        ac.mxfp4_mm_tensors(a, b, sb, y, A_scales=sa)
        A, B = (mx_ref.values(c.cpu().numpy(), s.cpu().numpy(), K) for c, s in ((a, sa), (b, sb)))
        tol = (K / 32 + 64) * (E * (np.abs(A) @ np.abs(B).T) + 2.0 ** -126)
        assert (np.abs(f64(y) - A @ B.T) <= tol).all(), total
    sa[:], sb[:] = 254, 254
    a[:], b[:] = 0x22, 0x22  # ones
    ac.mxfp4_mm_tensors(a, b, sb, y, A_scales=sa)
    assert (y == float("inf")).all()


def test_two_threads(t):
    """Two host threads on streams of their own, and on one."""
    import threading
    r = np.random.default_rng(12)
    M, N, K = 150, 400, 1500
    b, sb, _ = operand(t, r, N, K)
    xs = [t.from_numpy(r.normal(size=(M, K))).cuda().bfloat16() for _ in range(2)]
    want = []
    for x in xs:
        want.append(t.empty(M, N, device="cuda"))
        ac.mxfp4_mm_tensors(x, b, sb, want[-1])
    t.cuda.synchronize()
    one = t.cuda.Stream()
    for streams in ((t.cuda.Stream(), t.cuda.Stream()), (one, one)):
        outs, errors, start = [[t.empty(M, N, device="cuda") for _ in range(20)] for _ in xs], [], threading.Barrier(2)
        t.cuda.synchronize()

        def work(x, ys, stream):
            try:
                t.cuda.set_device(0)
                start.wait()
                for y in ys:
                    ac.mxfp4_mm_tensors(x, b, sb, y, stream=stream.cuda_stream)
            except Exception as e:  # noqa: BLE001
                errors.append(e)

        threads = [threading.Thread(target=work, args=job) for job in zip(xs, outs, streams)]
        for th in threads:
            th.start()
        for th in threads:
            th.join()
        t.cuda.synchronize()
        assert not errors, errors
        for ys, w in zip(outs, want):
            assert all(t.equal(y, w) for y in ys)


def test_refuses_tensors(t):
    r = np.random.default_rng(8)
    b, sb, _ = operand(t, r, 6, 40)
    a, sa, _ = operand(t, r, 4, 40)
    x, y = t.randn(4, 40, device="cuda"), t.empty(4, 6, device="cuda")
    c, s = t.empty(4, 32, dtype=t.uint8, device="cuda"), t.empty(4, 2, dtype=t.uint8, device="cuda")
    for bad in (lambda: ac.mxfp4_quantize_tensors(x.double(), c, s), lambda: ac.mxfp4_quantize_tensors(x, c.float(), s),
                lambda: ac.mxfp4_dequantize_tensors(c, s, x.int()),
                lambda: ac.mxfp4_mm_tensors(x.int(), b, sb, y),
                lambda: ac.mxfp4_mm_tensors(a, b, sb, y, A_scales=sa.float()),
                lambda: ac.mxfp4_mm_tensors(x, b, sb, y, bias=t.zeros(6, device="cuda").half())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: ac.mxfp4_quantize_tensors(x, c[:, :31], s), lambda: ac.mxfp4_quantize_tensors(x, c, s[:3]),
                lambda: ac.mxfp4_quantize_tensors(x[:, ::2], c[:, :16], s[:, :1]),
                lambda: ac.mxfp4_quantize_tensors(x.cpu(), c, s),
                lambda: ac.mxfp4_quantize_tensors(x, c.cpu(), s),
                lambda: ac.mxfp4_dequantize_tensors(c, s, x[:3]),
                lambda: ac.mxfp4_mm_tensors(x[:, :30], b, sb, y), lambda: ac.mxfp4_mm_tensors(x, b, sb, y[:, :5]),
                lambda: ac.mxfp4_mm_tensors(x, b[:, :16], sb, y), lambda: ac.mxfp4_mm_tensors(a[:, :16], b, sb, y, A_scales=sa),
                lambda: ac.mxfp4_gated_mm_tensors(x, b, sb, b[:5], sb, y),
                lambda: ac.mxfp4_gated_mm_tensors(x, b, sb, b, sb, y, act="relu")):
        with pytest.raises(ValueError):
            bad()
