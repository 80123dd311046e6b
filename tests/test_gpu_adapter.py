"""Low-rank adapters beside a shared projection on the GPU against the 64-bit
formula.

Tolerances. e = 2^-24, u = 2^-8 (bf16), 2^-11 (fp16). The shared product and
the adapters' first product are summed in fp32 over K: K e sum|a b|. T is
scaled (e) and, at worst, rounded to 16 bits: u |T| (fp16: 2^-25 where it is
subnormal). The second product adds R + 1 sums to it. With |S| the sum of
absolute values of everything that enters an element:

    (K + R + 3) e |S| + u (|T| |up|) + what T's K e sum|x down| becomes through
    |up|, then one rounding to Y's type

and the 2-norm of the whole error stays within 2 u of the output's (two
independent roundings of at most u / sqrt(3) each, and the fp32 sums).
"""
import numpy as np
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


class Problem:
    def __init__(self, t, M, N, K, n, R, dtype=None, out=None, col=True, pad=0, off=0, scale=True, bias=True, index=None,
                 seed=0):
        self.t, self.M, self.N, self.K, self.n, self.R = t, M, N, K, n, R
        self.dt = dtype or t.bfloat16
        self.u = 2.0 ** -8 if self.dt == t.bfloat16 else 2.0 ** -11
        self.tiny = 0.0 if self.dt == t.bfloat16 else 2.0 ** -25
        self.g = t.Generator(device="cuda").manual_seed(seed + M + 3 * N + 5 * K + 7 * R)
        self.pad, self.off = pad, off
        self.x = self.mat(M, K, 1.0)
        self.w = self.mat(N, K, K ** -0.5).t() if col else self.mat(K, N, K ** -0.5)
        self.down = self.stack(n, R, K, K ** -0.5)
        self.up = self.stack(n, N, R, R ** -0.5 if R else 1.0)
        self.scale = t.rand(n, device="cuda", generator=self.g) + 0.5 if scale else None
        self.bias = t.randn(N, device="cuda", generator=self.g) if bias else None
        if index is None:
            index = t.randint(-1, n, (M,), device="cuda", generator=self.g) if n else t.full((M,), -1, device="cuda")
        self.index = t.as_tensor(index, device="cuda").to(t.int32)
        self.odt = out or self.dt
        ld = N + pad
        self.buf = t.full((M * ld + off + 64,), 555.0, dtype=self.odt, device="cuda")
        self.y = self.buf[off:off + M * ld].view(M, ld)[:, :N]

    def mat(self, rows, cols, scale):
        t, ld = self.t, cols + self.pad
        buf = t.full((rows * ld + self.off,), float("nan"), dtype=self.dt, device="cuda")
        v = buf[self.off:].view(rows, ld)[:, :cols]
        v.copy_(t.randn(rows, cols, device="cuda", generator=self.g) * scale)
        return v

    def stack(self, n, rows, cols, scale):
        """A stack whose matrices lie apart, with NaN between the rows."""
        return self.mat(n * (rows + (1 if self.pad else 0)), cols, scale).unflatten(
            0, (n, rows + (1 if self.pad else 0)))[:, :rows]

    def run(self):
        return ac.adapter_mm_tensors(self.x, self.w, self.down, self.up, self.index, self.y, scale=self.scale,
                                     bias=self.bias)

    def check(self):
        t = self.t
        x, w = self.x.double(), self.w.double()
        ref, mag = x @ w, x.abs() @ w.abs()
        if self.bias is not None:
            ref += self.bias.double()
            mag += self.bias.double().abs()
        extra = t.zeros_like(ref)
        for a in range(self.n):
            rows = (self.index == a).nonzero().view(-1)
            if rows.numel() == 0 or self.R == 0:
                continue
            d, p = self.down[a].double(), self.up[a].double()
            s = self.scale[a].double() if self.scale is not None else 1.0
            tt, tm = s * (x[rows] @ d.t()), s * (x[rows].abs() @ d.t().abs())
            ref[rows] += tt @ p.t()
            mag[rows] += tm @ p.t().abs()
            extra[rows] += (self.u * tt.abs() + self.tiny + self.K * E * tm) @ p.t().abs()
        tol = (self.K + self.R + 3) * E * mag + extra
        f32 = self.odt == t.float32
        u = E if f32 else self.u
        tol = tol + u * (ref.abs() + tol) + (0.0 if f32 else self.tiny) + 1e-30
        got = self.y.double()
        assert t.isfinite(got).all()
        worst = ((got - ref).abs() / tol).max().item() if got.numel() else 0.0
        assert worst <= 1.0, worst
        if got.numel() >= 1000:
            rel = ((got - ref).norm() / ref.norm()).item()
            assert rel <= 2 * self.u, rel
        keep = t.ones_like(self.buf, dtype=t.bool)
        ld = self.N + self.pad
        keep[self.off:self.off + self.M * ld].view(self.M, ld)[:, :self.N] = False
        assert (self.buf[keep] == 555.0).all()


# M, N, K, adapters, rank
SIZES = [(1, 256, 512, 1, 16), (3, 512, 256, 8, 8), (16, 4096, 1024, 16, 16), (40, 1000, 512, 5, 24), (64, 264, 4096, 32, 64),
         (130, 512, 520, 3, 4), (300, 2048, 512, 70, 16), (1100, 1024, 1024, 9, 33), (2048, 2048, 512, 8, 16),
         (2100, 4096, 256, 4, 64), (4096, 4096, 320, 40, 16), (20000, 256, 128, 12, 20),
         (2040, 4096, 1024, 6, 16), (4000, 8192, 512, 30, 24), (1285, 5952, 1408, 6, 16)]


def test_sizes_cover_the_kernels(t):
    ks = set()
    for M, N, K, _, _ in SIZES:
        ks |= {k.split(" x")[0] for k in ac.adaptcore_adapter_kernels(M, N, K)}
    assert {"k_adapter<128, 128>", "k_adapter<128, 128, 3>", "k_adapter<256, 256>", "k_adapter_sum",
            "k_multi<32, 128>"} <= ks, ks


@pytest.mark.parametrize("kind", ["bf16_c", "f16_r", "bf16_r_f32", "f16_c_f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_adapters(t, size, kind):
    p = Problem(t, *size, dtype=t.float16 if kind.startswith("f16") else t.bfloat16, col="_c" in kind,
                out=t.float32 if kind.endswith("f32") else None)
    p.run()
    p.check()


@pytest.mark.parametrize("col", [True, False])
@pytest.mark.parametrize("size", [(1, 1, 1, 1, 1), (5, 77, 33, 3, 5), (17, 130, 101, 4, 7), (200, 515, 333, 6, 9),
                                  (900, 301, 250, 2, 17), (30, 256, 512, 4, 16)], ids=lambda s: "x".join(map(str, s)))
def test_odd_sizes_and_pitches(t, size, col):
    """Sizes, pitches and addresses that are not whole chunks, and NaN in
    every operand between its rows."""
    p = Problem(t, *size, col=col, pad=3, off=1)
    p.run()
    p.check()


@pytest.mark.parametrize("M", [16, 700, 2048])
def test_indices(t, M):
    """One adapter for all rows, none for any, values outside, runs of rows,
    the last adapter alone."""
    n = 6
    for index in (t.full((M,), 2), t.full((M,), -1), t.full((M,), n), t.full((M,), 2 ** 31 - 1), t.full((M,), -2 ** 31),
                  t.arange(M) // max(1, M // 11) - 2, t.where(t.arange(M) == M - 1, n - 1, -1),
                  (t.arange(M) % (2 * n)) - 3):
        p = Problem(t, M, 512, 256, n, 16, index=index)
        p.run()
        p.check()


def test_without(t):
    """No scale, no bias, no adapters, rank 0, K 0, no rows."""
    for size, kw in (((40, 256, 128, 4, 16), dict(scale=False)), ((700, 512, 128, 4, 16), dict(bias=False)),
                     ((40, 256, 128, 0, 16), dict(scale=False)), ((700, 512, 128, 0, 16), dict()),
                     ((40, 256, 128, 3, 0), dict()), ((700, 512, 128, 3, 0), dict(bias=False))):
        p = Problem(t, *size, **kw)
        p.run()
        p.check()
    for M in (5, 700):
        x, w = t.empty(M, 0, device="cuda", dtype=t.float16), t.empty(0, 256, device="cuda", dtype=t.float16)
        y, bias = t.empty(M, 256, device="cuda", dtype=t.float16), t.randn(256, device="cuda")
        ac.adapter_mm_tensors(x, w, t.empty(2, 4, 0, device="cuda", dtype=t.float16),
                              t.ones(2, 256, 4, device="cuda", dtype=t.float16),
                              t.zeros(M, device="cuda", dtype=t.int32), y, bias=bias)
        assert t.equal(y, bias.half().expand(M, 256))
    p = Problem(t, 0, 64, 32, 2, 4)
    p.run()


def test_no_adapters_needs_no_index(t):
    for M in (5, 700):
        x, w = t.randn(M, 64, device="cuda").half(), t.randn(64, 256, device="cuda").half()
        y = t.empty(M, 256, device="cuda", dtype=t.float16)
        ac.adaptcore_adapter_matmul(M, 256, 64, ac.AC_F16_F16OUT, 0, x.data_ptr(), 64, w.data_ptr(), 256, 0, 0, 0, 1, 0,
                                    0, 1, 0, 0, 0, 0, y.data_ptr(), 256, t.cuda.current_stream().cuda_stream)
        ref = x.double() @ w.double()
        # 64 terms of order one: the sum's fp32 error and one rounding of values below 64
        assert (y.double() - ref).abs().max() <= 2.0 ** -11 * 64


def test_oracle_agrees(t):
    p = Problem(t, 20, 40, 24, 3, 5)
    p.run()
    ref = ffn_ref.adapter_mm(*(v.double().cpu().numpy() for v in (p.x, p.w, p.down, p.up)), p.index.cpu().numpy(),
                             p.scale.double().cpu().numpy(), p.bias.double().cpu().numpy())
    assert np.abs(p.y.double().cpu().numpy() - ref).max() <= 2 * p.u * np.abs(ref).max()


def test_non_finite_stays_alone(t):
    """A row with a NaN, and an adapter with NaN weights that some rows use:
    the other rows keep their results, in tiles shared with them too."""
    for M, K, R in ((24, 128, 16), (600, 100, 12), (2048, 128, 20)):
        index = t.arange(M) % 5 - 1
        p = Problem(t, M, 512, K, 4, R, index=index)
        clean = p.run().clone()
        p.x[7, K - 1] = float("nan")
        p.down[2, R - 1, 0] = float("nan")
        p.up[3, 5, R - 1] = float("inf")
        p.run()
        rows = (p.index != 2) & (p.index != 3)
        rows[7] = False
        assert t.equal(p.y[rows], clean[rows])
        assert t.isnan(p.y[p.index == 2]).all() and t.isnan(p.y[7]).all()
        others = t.arange(512, device="cuda") != 5
        threes = p.index == 3
        threes[7] = False
        assert t.equal(p.y[threes][:, others], clean[threes][:, others])


def test_same_bits_and_other_stream(t):
    for size in ((16, 1024, 1024, 8, 16), (900, 1024, 256, 8, 16)):
        outs = []
        for s in (t.cuda.current_stream(), t.cuda.Stream()):
            p = Problem(t, *size)
            t.cuda.synchronize()
            with t.cuda.stream(s):
                p.run()
            s.synchronize()
            outs.append(p.y.clone())
        assert t.equal(*outs)


@pytest.mark.parametrize("size", [(9, 515, 333, 4, 7), (64, 2048, 1024, 8, 16), (700, 512, 256, 8, 16)],
                         ids=lambda s: "x".join(map(str, s)))
def test_graph_replays(t, size):
    """The indices are read when the graph runs: new ones with every replay."""
    p = Problem(t, *size)
    s = t.cuda.Stream()
    ac.adaptcore_reserve_workspace(s.cuda_stream, ac.adaptcore_adapter_workspace(*size[:3], size[4]))
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph, stream=s):
        p.run()
    for i in range(4):
        p.x.copy_(t.randn(p.M, p.K, device="cuda"))
        p.index.copy_(t.randint(-1, p.n, (p.M,), device="cuda"))
        t.cuda.synchronize()
        graph.replay()
        t.cuda.synchronize()
        got = p.y.clone()
        p.y.fill_(0)
        p.run()
        t.cuda.synchronize()
        assert t.equal(got, p.y), i


def test_refuses_tensors(t):
    p = Problem(t, 4, 16, 24, 2, 8)
    ok = (p.x, p.w, p.down, p.up, p.index, p.y)

    def sub(i, v):
        a = list(ok)
        a[i] = v
        return a

    for a in (sub(0, p.x.float()), sub(1, p.w.half()), sub(2, p.down.half()), sub(3, p.up.float()),
              sub(4, p.index.long()), sub(5, p.y.half())):
        with pytest.raises(TypeError):
            ac.adapter_mm_tensors(*a)
    for a in (sub(1, p.w[:20]), sub(2, p.down[0]), sub(2, p.down.transpose(1, 2)), sub(3, p.up.transpose(1, 2)),
              sub(4, p.index[:3]), sub(5, p.y[:, :8]), sub(3, p.up[:1]), sub(4, p.index.cpu())):
        with pytest.raises(ValueError):
            ac.adapter_mm_tensors(*a)
    with pytest.raises(ValueError):
        ac.adapter_mm_tensors(*ok, scale=t.ones(3, device="cuda"))
    with pytest.raises(ValueError):
        ac.adapter_mm_tensors(*ok, bias=t.ones(24, device="cuda"))


@pytest.mark.parametrize("scale", [1e6, 1.0, 1e-7])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("size", [(1, 256, 512, 1, 16), (16, 1000, 264, 5, 33), (64, 520, 1024, 9, 8)],
                         ids=lambda s: "x".join(map(str, s)))
def test_few_rows_keep_t_in_32_bits(t, size, kind, scale):
    """T far beyond fp16's range and far below its smallest values, with `up`
    the other way, fp32 outputs. T's sum is within K e sum|x down| scale; what
    its two 16-bit terms lose is 2^-16 of each value (bf16) or 2^-22 of the
    row's greatest (fp16)."""
    M, N, K, n, R = size
    p = Problem(t, *size, dtype=t.float16 if kind == "f16" else t.bfloat16, out=t.float32, index=t.arange(M) % n)
    p.scale.mul_(scale)
    p.up.mul_(min(1.0 / scale, 1000.0))
    p.run()
    x, w = p.x.double(), p.w.double()
    ref = x @ w + p.bias.double()
    tol = (K + 3) * E * (x.abs() @ w.abs() + p.bias.double().abs())
    for a in range(n):
        rows = (p.index == a).nonzero().view(-1)
        d, u, s = p.down[a].double(), p.up[a].double(), p.scale[a].double()
        tt, tm = s * (x[rows] @ d.t()), s * (x[rows].abs() @ d.t().abs())
        lost = 2.0 ** -22 * tt.abs().amax(1, keepdim=True).expand_as(tt) if kind == "f16" else 2.0 ** -16 * tt.abs()
        ref[rows] += tt @ u.t()
        tol[rows] += (K * E * tm + lost + (2 * R + 3) * E * tt.abs()) @ u.t().abs()
    got = p.y.double()
    assert t.isfinite(got).all()
    worst = ((got - ref).abs() / (tol + E * (ref.abs() + tol))).max().item()
    assert worst <= 1.0, worst


def test_one_row_of_any_stride(t):
    """One token, and adapters of rank one, whose only rows may lie at any
    stride."""
    far = 2 ** 23 + 64
    p = Problem(t, 1, 256, 128, 2, 1, index=t.ones(1))
    p.run()
    x, y = (t.empty(1, far, device="cuda", dtype=p.dt)[:, 8:8 + n] for n in (128, 256))
    x.copy_(p.x)
    down = t.empty(2, 1, far, device="cuda", dtype=p.dt)[:, :, :128].copy_(p.down)
    ac.adapter_mm_tensors(x, p.w, down, p.up, p.index, y, scale=p.scale, bias=p.bias)
    assert t.equal(y, p.y)


# K split over launches for more rows than T is made beside, and ranks past 64.
# M, N, K, adapters, rank, what runs
SPLIT = [(300, 512, 4096, 70, 24, "k_shrink;k_multi<32, 128> x5;k_adapter_sum"),
         (400, 4096, 8192, 12, 20, "k_shrink;k_multi<128, 256> x4;k_adapter_sum"),
         (1000, 512, 4096, 30, 16, "k_shrink;k_multi<32, 128> x2;k_adapter_sum"),
         (16500, 128, 8192, 9, 12, "k_shrink;k_multi<128, 128> x3;k_adapter_sum"),
         (16, 1024, 2048, 4, 65, "k_shrink;k_multi<32, 128> x4;k_adapter_sum"),
         (64, 520, 1024, 9, 200, "k_shrink;k_multi<32, 128> x2;k_adapter_sum"),
         (1, 256, 512, 2, 4096, "k_shrink;k_multi<32, 128>;k_adapter_sum"),
         (130, 512, 520, 3, 256, "k_shrink;k_adapter<128, 128, 3>"),
         (700, 1024, 512, 5, 129, "k_shrink;k_adapter<128, 128, 3>"),
         (2100, 4096, 256, 3, 100, "k_shrink;k_adapter<128, 128>")]


@pytest.mark.parametrize("kind", ["bf16_c", "f16_r", "f16_c_f32"])
@pytest.mark.parametrize("size", SPLIT, ids=lambda s: "x".join(map(str, s[:5])))
def test_split_products_and_high_ranks(t, size, kind):
    M, N, K, n, R, kernels = size
    assert ";".join(ac.adaptcore_adapter_kernels(M, N, K, R)) == kernels
    # runs of rows and single ones of every adapter, some rows without
    index = t.where(t.arange(M) < M // 2, t.arange(M) // 37 % (n + 1) - 1, t.arange(M) % (n + 1) - 1)
    p = Problem(t, M, N, K, n, R, dtype=t.float16 if kind.startswith("f16") else t.bfloat16, col="_c" in kind,
                out=t.float32 if kind.endswith("f32") else None, index=index)
    before = ac.adaptcore_stats()["launches"]
    p.run()
    assert ac.adaptcore_stats()["launches"] - before == len(kernels.split(";"))
    p.check()


def test_more_rows_than_one_launch_of_sums_takes(t):
    """The most rows there may be, misaligned (the product on its own plan),
    with the last adapter in the last row."""
    M = 2 ** 22 - 1
    index = t.full((M,), -1)
    index[0], index[M - 64:] = 0, 1
    p = Problem(t, M, 9, 9, 2, 5, pad=1, off=1, index=index)
    p.run()
    p.check()


def test_launches_of_few_rows(t):
    for R, count in ((16, 2), (64, 2), (65, 3)):
        p = Problem(t, 16, 512, 1024, 3, R)
        assert len(ac.adaptcore_adapter_kernels(16, 512, 1024, R)) == count
        before = ac.adaptcore_stats()["launches"]
        p.run()
        assert ac.adaptcore_stats()["launches"] - before == count
        p.check()
