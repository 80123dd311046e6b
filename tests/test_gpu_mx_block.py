"""The 4-bit operators and the joint as a model uses them: a stack of blocks served
in 4 bits, each call against the 64-bit form of what it was given, and a block
between two joints trained.

Tolerances, with e = 2^-24: codes and scales equal those of the norm as it is
stored. Products as in the operators' own tests: e (K / 32 + 64) of the sum of the
terms' magnitudes. silu(g) u is off by 1.1 |u| dg + |silu(g)| du (the slope of silu
is below 1.1) and 8 e. The joint's R is off by 2 e before it is stored; its N as in
the joint's own tests. Results stored in bfloat16 add 2^-8.
"""
import importlib.util
import os

import numpy as np
import pytest

import paper_2608_10803_amd as ac
from oracle import join_ref, mx_ref

pytestmark = pytest.mark.gpu

E, U = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def example():
    import torch
    assert torch.cuda.is_available()
    ac.adaptcore_init()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "feed_forward_block.py")
    spec = importlib.util.spec_from_file_location("feed_forward_block", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def f64(x):
    return x.detach().double().cpu().numpy()


def near(got, ref, tol, label):
    err, tol = np.abs(f64(got) - ref), tol + U * (np.abs(ref) + tol) + 1e-300
    assert (err <= tol).all(), (label, np.max(err / tol))


def product_tol(a, b):
    return E * (a.shape[1] / 32 + 64) * (np.abs(a) @ np.abs(b).T)


def norm_tol(f, w, b):
    """Error of the layer norm's output, of a forward pass f of join_ref."""
    v, xh, r = f["r"], np.abs(f["xh2"]), f["r2"][:, None]
    d = 2 * E * np.abs(v)
    d = d + d.mean(1)[:, None] + 96 * E * np.abs(v).mean(1)[:, None] + 2 * E * (np.abs(v) + np.abs(f["m2"])[:, None])
    dx = r * d + xh * ((xh * d).mean(1)[:, None] * r + 101 * E)
    return dx * np.abs(w) + 3 * E * (xh * np.abs(w) + np.abs(b))


@pytest.mark.parametrize("rows,dim,hidden", [(1, 256, 704), (16, 160, 417), (33, 256, 704), (257, 96, 1000), (0, 64, 96)])
def test_a_stack_in_4_bits(example, rows, dim, hidden):
    import torch
    blocks = [example.Block(dim, hidden, seed=20 + i) for i in range(3)]
    g = torch.Generator(device="cuda").manual_seed(rows)
    for b in blocks:
        b.master[0].uniform_(0.5, 1.5, generator=g)
        b.master[1].normal_(generator=g)
    stack = example.Stack4(blocks, rows)
    x = torch.randn(rows, dim, device="cuda", generator=g).bfloat16()
    want = stack(x.clone())
    # the same with what lies between the calls looked at: N stored too, the
    # hidden rows quantised by a call of their own
    r, y, n = x.clone(), torch.empty_like(x), torch.empty_like(x)
    h = torch.empty(rows, hidden, device="cuda", dtype=x.dtype)
    for i, ((wg, sg), (wu, su), (wd, sd)) in enumerate(stack.matrices):
        w, b = blocks[i].master[:2]
        codes, scales = stack.empty4(rows, dim)
        before = r.clone()
        ac.residual_norm_tensors(r, y if i else None, r if i else None, n, norm="layer", post=False, weight=w, bias=b,
                                 codes=codes, code_scales=scales)
        ref = join_ref.forward(f64(before), f64(y) if i else None, "layer", False, w2=f64(w), b2=f64(b))
        near(r, ref["r"], 2 * E * np.abs(ref["r"]), "r")
        near(n, ref["n"], norm_tol(ref, f64(w), f64(b)), "n")
        c, s = ac.mxfp4_quantize_tensors(n, *stack.empty4(rows, dim))
        assert torch.equal(codes, c) and torch.equal(scales, s)
        ac.mxfp4_gated_mm_tensors(codes, wg, sg, wu, su, h, A_scales=scales)
        a, mg, mu = (mx_ref.values(c.cpu().numpy(), s.cpu().numpy(), dim) for c, s in ((codes, scales), (wg, sg), (wu, su)))
        ref, gate, up = mx_ref.gated(a, mg, mu, "silu")
        silu = np.abs(gate) / (1 + np.exp(-gate))
        near(h, ref, 1.1 * np.abs(up) * product_tol(a, mg) + silu * product_tol(a, mu) + 8 * E * np.abs(ref), "h")
        hc, hs = ac.mxfp4_quantize_tensors(h, *stack.empty4(rows, hidden))
        ac.mxfp4_mm_tensors(hc, wd, sd, y, A_scales=hs)
        a, m = (mx_ref.values(c.cpu().numpy(), s.cpu().numpy(), hidden) for c, s in ((hc, hs), (wd, sd)))
        near(y, mx_ref.product(a, m), product_tol(a, m), "y")
    ac.residual_norm_tensors(r, y, r, post=False)
    assert torch.equal(r, want)


@pytest.mark.parametrize("rows", [1, 20, 300])
def test_a_stack_replayed(example, rows):
    import torch
    out, _ = example.serve4(rows=rows, replays=4)
    assert len(out) == 4
    for a, b in out:
        assert torch.equal(a, b) and bool(a.isfinite().all())


@pytest.mark.parametrize("norm,gate_rows", [("rms", 0), ("layer", 3)])
def test_a_block_between_two_joints_trained(example, norm, gate_rows):
    """R1, N1 = joint(x, a), y = gated block of N1, R2, N2 = joint(R1, y): gradients
    along random directions against central differences of the 64-bit form."""
    import torch
    rows, dim, hidden = 60, 64, 176
    block = example.Block(dim, hidden, seed=5)
    g = torch.Generator(device="cuda").manual_seed(6)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    def like(v, n=1):
        return [torch.empty_like(v) for _ in range(n)]

    x, dr2 = normal(rows, dim), normal(rows, dim)  # the residual stream in 32 bits
    a, dn2 = normal(rows, dim).bfloat16(), normal(rows, dim).bfloat16()
    w = [1 + 0.3 * normal(dim) for _ in range(4)]  # of the post and the next norm of either joint
    gate = 1 + 0.3 * normal(gate_rows, dim) if gate_rows else None
    r1, r2 = like(x, 2)
    n1, y, n2 = like(a, 3)
    h, gt, up = (torch.empty(rows, hidden, device="cuda", dtype=a.dtype) for _ in range(3))
    s1, s2 = (torch.empty(rows, 4, device="cuda") for _ in range(2))
    ac.residual_norm_tensors(x, a, r1, n1, norm=norm, post_weight=w[0], gate=gate, weight=w[1], stats=s1)
    ac.gated_ffn_tensors(n1, *block.views(block.matrix), h, y, gate=gt, up=up)
    ac.residual_norm_tensors(r1, y, r2, n2, norm=norm, post_weight=w[2], weight=w[3], stats=s2)
    dr1, dx = like(x, 2)
    dy, dn1, da = like(a, 3)
    dw, dgate = like(w[0], 4), None if gate is None else torch.empty_like(gate)
    ac.residual_norm_backward_tensors(dr2, dn2, r1, y, s2, dr1, dy, norm=norm, post_weight=w[2], weight=w[3],
                                      dpost_weight=dw[2], dweight=dw[3])
    ac.gated_ffn_backward_tensors(dy, n1, *block.views(block.matrix), gt, up, h, dX=dn1,
                                  **dict(zip(("dWg", "dWu", "dWd"), block.views(block.grad[2:]))))
    ac.residual_norm_backward_tensors(dr1, dn1, x, a, s1, dx, da, norm=norm, post_weight=w[0], gate=gate, weight=w[1],
                                      dpost_weight=dw[0], dgate=dgate, dweight=dw[1])
    at = [v.double() for v in [x, a] + w + block.matrix] + ([] if gate is None else [gate.double()])

    def normed(v, weight):
        if norm == "layer":
            v = v - v.mean(1, keepdim=True)
        return v * (v.pow(2).mean(1, keepdim=True) + 1e-5).rsqrt() * weight

    def loss(x, a, p1, q1, p2, q2, wg, wu, wd, gate=None):
        p = normed(a, p1)
        r = x + (p if gate is None else torch.repeat_interleave(gate, rows // gate_rows, 0) * p)
        n = normed(r, q1)
        t = n @ wg.t()
        r = r + normed((t * torch.sigmoid(t) * (n @ wu.t())) @ wd.t(), p2)
        return (r * dr2.double()).sum() + (normed(r, q2) * dn2.double()).sum()

    for i, grad in enumerate([dx, da] + dw + block.grad[2:] + ([] if gate is None else [dgate])):
        v = torch.randn(at[i].shape, device="cuda", dtype=torch.float64, generator=g)
        hi, lo = list(at), list(at)
        hi[i], lo[i] = at[i] + 1e-5 * v, at[i] - 1e-5 * v
        d = (loss(*hi) - loss(*lo)) / 2e-5
        # ten roundings to bfloat16 on the way (N1, gate, up, h, y; dy, those of the
        # block's backward pass, dN1, da), five standard deviations of a direction
        assert abs((grad.double() * v).sum() - d) <= 5 * 10 * U * grad.double().norm(), i
