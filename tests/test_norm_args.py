"""What layer norm refuses, and its sizes that need no launch (no GPU)."""
import pytest

import paper_2608_10803_amd as ac

F32, BF16, F16 = ac.AC_TYPE_F32, ac.AC_TYPE_BF16, ac.AC_TYPE_F16
P = 1 << 20  # an aligned address that is never read


def forward(**k):
    a = dict(rows=4, cols=8, type=BF16, weight_type=F32, X=P, ldx=8, weight=P, bias=P, eps=1e-5, Y=2 * P, ldy=8,
             mean=0, rstd=0)
    a.update(k)
    return ac.adaptcore_layer_norm(**a)


def backward(**k):
    a = dict(rows=4, cols=8, type=BF16, weight_type=F32, dY=P, lddy=8, X=P, ldx=8, weight=P, mean=P, rstd=P, dX=2 * P,
             lddx=8, dweight=P, dbias=P)
    a.update(k)
    return ac.adaptcore_layer_norm_backward(**a)


BOTH = [dict(rows=-1), dict(rows=1 << 31), dict(cols=-1), dict(cols=1 << 30, ldx=1 << 30), dict(ldx=7), dict(X=P + 1),
        dict(weight=P + 2), dict(X=0), dict(type=F32, X=P + 2), dict(rstd=P + 2)]


@pytest.mark.parametrize("bad", BOTH + [dict(ldy=7), dict(Y=0), dict(Y=P + 1), dict(eps=-1e-9), dict(eps=float("nan")),
                                        dict(eps=float("inf")), dict(bias=P + 1), dict(mean=P + 1)])
def test_forward_refuses(bad):
    with pytest.raises(ac.AdaptCoreError) as e:
        forward(**bad)
    assert e.value.status == ac.AC_ERR_INVALID_VALUE


@pytest.mark.parametrize("bad", BOTH + [dict(lddy=7), dict(lddx=7), dict(dY=0), dict(dX=0), dict(mean=0), dict(rstd=0),
                                        dict(dweight=P + 2), dict(dbias=P + 1), dict(dX=P + 1)])
def test_backward_refuses(bad):
    with pytest.raises(ac.AdaptCoreError) as e:
        backward(**bad)
    assert e.value.status == ac.AC_ERR_INVALID_VALUE


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("bad", [dict(type=3), dict(type=-1), dict(weight_type=F16), dict(type=F32, weight_type=BF16),
                                 dict(weight_type=7)])
def test_types(call, bad):
    with pytest.raises(ac.AdaptCoreError) as e:
        call(**bad)
    assert e.value.status == ac.AC_ERR_UNSUPPORTED


def test_nothing_to_do():
    forward(rows=0, X=0, Y=0)
    forward(cols=0, ldx=1, ldy=1, X=0, Y=0)
    backward(cols=0, lddy=1, ldx=1, lddx=1, dY=0, X=0, dX=0)
    backward(rows=0, dweight=0, dbias=0, dY=0, X=0, dX=0, mean=0, rstd=0)


def test_workspace():
    assert ac.adaptcore_layer_norm_backward_workspace(0, 100) == 0
    assert ac.adaptcore_layer_norm_backward_workspace(1, 100) == 800
    assert ac.adaptcore_layer_norm_backward_workspace(10 ** 6, 4096) <= 64 << 20
    assert ac.adaptcore_layer_norm_backward_workspace(10 ** 6, 1 << 20) == 32 * 2 * (1 << 20) * 4
    with pytest.raises(ac.AdaptCoreError):
        ac.adaptcore_layer_norm_backward_workspace(-1, 4)
