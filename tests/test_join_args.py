"""What the residual joint refuses, and its sizes that need no launch (no
GPU)."""
import pytest

import paper_2608_10803_amd as ac

F32, BF16, F16 = ac.AC_TYPE_F32, ac.AC_TYPE_BF16, ac.AC_TYPE_F16
P = 1 << 20  # an aligned address that is never read


def joint(**k):
    a = dict(rows=4, cols=40, residual_type=BF16, type=BF16, weight_type=F32, norm=0, post=1, pre=1, scale=1.0, eps=1e-5,
             X=P, ldx=40, Y=P, ldy=40, post_weight=P, post_bias=P, gate=P, gate_rows=2, ld_gate=40, weight=P, bias=P)
    a.update({n: k[n] for n in list(k) if n in a})
    return ac._lib.ResidualNorm(**a), {n: v for n, v in k.items() if n not in a}


def forward(**k):
    p, rest = joint(**k)
    a = dict(R=2 * P, ldr=40, N=3 * P, ldn=40)
    a.update(rest)
    return ac.adaptcore_residual_norm(p, **a)


def backward(**k):
    p, rest = joint(**k)
    a = dict(dR=P, lddr=40, dN=P, lddn=40, stats=P, dX=2 * P, lddx=40, dY=3 * P, lddy=40, dpost_weight=P, dpost_bias=P,
             dgate=P, ld_dgate=40, dweight=P, dbias=P)
    a.update(rest)
    return ac.adaptcore_residual_norm_backward(p, **a)


def status(call, **k):
    with pytest.raises(ac.AdaptCoreError) as e:
        call(**k)
    return e.value.status


BOTH = [dict(rows=-1), dict(rows=1 << 31), dict(cols=-1), dict(cols=1 << 30), dict(ldx=39), dict(ldy=39),
        dict(ld_gate=39), dict(X=0), dict(X=P + 1), dict(Y=P + 1), dict(gate=P + 2), dict(post_weight=P + 2),
        dict(weight=P + 1), dict(gate_rows=3), dict(gate_rows=0), dict(gate_rows=-1), dict(eps=-1.0),
        dict(eps=float("nan")), dict(scale=float("inf")), dict(Y=0), dict(Y=0, post=0, post_weight=0, post_bias=0),
        dict(post=0), dict(pre=0, weight=P)]


@pytest.mark.parametrize("bad", BOTH + [dict(ldr=39), dict(ldn=39), dict(R=2 * P + 1), dict(N=3 * P + 1),
                                        dict(N=0), dict(pre=0, weight=0, bias=0),
                                        dict(pre=0, weight=0, bias=0, N=0, R=0), dict(codes=P),
                                        dict(codes=P, scales=P, ld_codes=31, ld_scales=2),
                                        dict(codes=P, scales=P, ld_codes=32, ld_scales=1), dict(stats=P + 2)])
def test_forward_refuses(bad):
    assert status(forward, **bad) == ac.AC_ERR_INVALID_VALUE


@pytest.mark.parametrize("bad", BOTH + [dict(lddr=39), dict(lddn=39), dict(lddx=39), dict(lddy=39), dict(ld_dgate=39),
                                        dict(dR=P + 1), dict(dX=P + 1), dict(dgate=P + 2), dict(dweight=P + 1),
                                        dict(stats=0), dict(dN=0), dict(gate=0), dict(dN=0, dR=0, dweight=0, dbias=0),
                                        dict(post=0, post_weight=0, post_bias=0),
                                        dict(pre=0, weight=0, bias=0, dN=0)])
def test_backward_refuses(bad):
    assert status(backward, **bad) == ac.AC_ERR_INVALID_VALUE


def backward_apart(**k):
    """backward() with an address of its own for everything."""
    a = dict(X=4 * P, Y=5 * P, post_weight=6 * P, post_bias=7 * P, gate=8 * P, weight=9 * P, bias=10 * P, dR=11 * P, dN=12 * P,
             stats=13 * P, dX=2 * P, dY=3 * P, dpost_weight=14 * P, dpost_bias=15 * P, dgate=16 * P, dweight=17 * P, dbias=18 * P)
    a.update(k)
    return backward(**a)


@pytest.mark.parametrize("bad", [dict(dX=11 * P), dict(dX=12 * P), dict(dX=4 * P), dict(dX=5 * P), dict(dY=11 * P),
                                 dict(dY=12 * P), dict(dY=4 * P), dict(dY=5 * P), dict(dX=3 * P), dict(dgate=8 * P),
                                 dict(dgate=2 * P), dict(dgate=4 * P), dict(dX=8 * P), dict(dY=11 * P, dX=0),
                                 dict(dX=11 * P, dY=0, dgate=0)])
@pytest.mark.parametrize("cols", [40, 5, 9000])
def test_backward_refuses_outputs_over_inputs(bad, cols):
    """Of rows of any length, also where the kernel of some would not mind."""
    ld = {n: cols for n in ("cols", "ldx", "ldy", "ld_gate", "lddr", "lddn", "lddx", "lddy", "ld_dgate")}
    assert status(backward_apart, **bad, **ld) == ac.AC_ERR_INVALID_VALUE
    assert "must not lie over" in ac.adaptcore_last_error()


def test_backward_refuses_for_each_reason_alone():
    """With nothing over anything, so that no other refusal stands in."""
    for bad in (dict(lddr=39), dict(lddn=39), dict(lddx=39), dict(lddy=39), dict(ld_dgate=39), dict(dR=11 * P + 1),
                dict(dX=2 * P + 1), dict(dgate=16 * P + 2), dict(dweight=17 * P + 1), dict(stats=0), dict(dN=0), dict(gate=0),
                dict(post=0, post_weight=0, post_bias=0), dict(pre=0, weight=0, bias=0, dN=0)):
        assert status(backward_apart, **bad) == ac.AC_ERR_INVALID_VALUE, bad
        assert "must not lie over" not in ac.adaptcore_last_error(), bad


def test_nothing_lies_over_anything_where_there_is_nothing():
    """Empty matrices may have any addresses, the same ones too."""
    backward_apart(cols=0, ldx=1, ldy=1, ld_gate=1, lddr=1, lddn=1, lddx=1, lddy=1, ld_dgate=1, dX=11 * P)
    backward_apart(rows=0, gate_rows=1, dX=11 * P, dY=11 * P, dpost_weight=0, dpost_bias=0, dgate=0, dweight=0, dbias=0)


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("bad", [dict(type=3), dict(residual_type=F16), dict(weight_type=F16), dict(weight_type=-1),
                                 dict(norm=2), dict(type=F32, residual_type=BF16)])
def test_types(call, bad):
    assert status(call, **bad) == ac.AC_ERR_UNSUPPORTED


def test_nothing_to_do():
    forward(rows=0, X=0, gate_rows=1)
    forward(cols=0, ldx=1, ldy=1, ld_gate=1, ldr=1, ldn=1)
    backward(cols=0, ldx=1, ldy=1, ld_gate=1, lddr=1, lddn=1, lddx=1, lddy=1, ld_dgate=1)
    backward(rows=0, gate_rows=1, dpost_weight=0, dpost_bias=0, dgate=0, dweight=0, dbias=0)


def test_workspace():
    assert ac.adaptcore_residual_norm_backward_workspace(0, 100) == 0
    assert ac.adaptcore_residual_norm_backward_workspace(1, 100) >= 4 * 100 * 4
    assert ac.adaptcore_residual_norm_backward_workspace(10 ** 6, 4096, 1) <= 512 * 5 * 4096 * 4
    # a gate of every row has no partial sums
    assert ac.adaptcore_residual_norm_backward_workspace(4096, 4096, 4096) <= 512 * 4 * 4096 * 4
    with pytest.raises(ac.AdaptCoreError):
        ac.adaptcore_residual_norm_backward_workspace(10, 4, 3)
