"""What the 4-bit entry points refuse, and the sizes that need no launch (no
GPU)."""
import pytest

import paper_2608_10803_amd as ac

F32, BF16, F16, MX = ac.AC_TYPE_F32, ac.AC_TYPE_BF16, ac.AC_TYPE_F16, ac.AC_TYPE_MXFP4
P = 1 << 20  # an aligned address that is never read


def quantize(**k):
    a = dict(rows=4, cols=40, type=BF16, layout=0, X=P, ldx=40, codes=2 * P, ld_codes=32, scales=3 * P, ld_scales=2)
    a.update(k)
    return ac.adaptcore_mxfp4_quantize(**a)


def dequantize(**k):
    a = dict(rows=4, cols=40, type=BF16, codes=2 * P, ld_codes=32, scales=3 * P, ld_scales=2, Y=P, ldy=40)
    a.update(k)
    return ac.adaptcore_mxfp4_dequantize(**a)


def matmul(**k):
    a = dict(M=4, N=6, K=40, a_type=MX, A=P, lda=32, A_scales=P, ld_a_scales=2, B=P, ldb=32, B_scales=P, ld_b_scales=2,
             bias=0, out_type=BF16, Y=P, ldy=6)
    a.update(k)
    return ac.adaptcore_mxfp4_matmul(**a)


def gated(**k):
    a = dict(M=4, F=6, K=40, a_type=MX, A=P, lda=32, A_scales=P, ld_a_scales=2, Bg=P, Bu=P, ldb=32, Bg_scales=P,
             Bu_scales=P, ld_b_scales=2, activation=0, type=BF16, H=P, ldh=6)
    a.update(k)
    return ac.adaptcore_mxfp4_gated_matmul(**a)


def status(call, **k):
    with pytest.raises(ac.AdaptCoreError) as e:
        call(**k)
    return e.value.status


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=1 << 31), dict(cols=-1), dict(cols=1 << 31, ldx=1 << 31),
                                 dict(ldx=39), dict(ld_codes=31), dict(ld_scales=1), dict(X=0), dict(codes=0),
                                 dict(scales=0), dict(X=P + 1), dict(type=F32, X=P + 2), dict(layout=1, ldx=3)])
def test_quantize_refuses(bad):
    assert status(quantize, **bad) == ac.AC_ERR_INVALID_VALUE


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(cols=1 << 31, ldy=1 << 31), dict(ldy=39), dict(ld_codes=31),
                                 dict(ld_scales=1), dict(Y=0), dict(codes=0), dict(scales=0), dict(Y=P + 1)])
def test_dequantize_refuses(bad):
    assert status(dequantize, **bad) == ac.AC_ERR_INVALID_VALUE


@pytest.mark.parametrize("bad", [dict(M=-1), dict(N=1 << 31, ldy=1 << 31), dict(K=1 << 23), dict(lda=31),
                                 dict(ld_a_scales=1), dict(ldb=31), dict(ld_b_scales=1), dict(lda=1 << 23),
                                 dict(ldb=1 << 23), dict(ldy=5), dict(ldy=1 << 23), dict(A=0), dict(A_scales=0), dict(B=0),
                                 dict(B_scales=0), dict(Y=0), dict(Y=P + 1), dict(bias=P + 2), dict(a_type=BF16, lda=39),
                                 dict(a_type=BF16, lda=40, A=P + 1), dict(a_type=F32, lda=40, A=0)])
def test_matmul_refuses(bad):
    assert status(matmul, **bad) == ac.AC_ERR_INVALID_VALUE


@pytest.mark.parametrize("bad", [dict(F=-1), dict(Bu=0), dict(Bu_scales=0), dict(ldb=31), dict(H=0), dict(ldh=5)])
def test_gated_refuses(bad):
    assert status(gated, **bad) == ac.AC_ERR_INVALID_VALUE


@pytest.mark.parametrize("call,bad", [(quantize, dict(type=3)), (quantize, dict(layout=2)), (dequantize, dict(type=-1)),
                                      (matmul, dict(a_type=4)), (matmul, dict(out_type=3)), (gated, dict(type=3)),
                                      (gated, dict(activation=3))])
def test_unsupported(call, bad):
    assert status(call, **bad) == ac.AC_ERR_UNSUPPORTED


@pytest.mark.parametrize("call,bad", [(quantize, dict(cols=1 << 30, ldx=1 << 30)), (dequantize, dict(cols=1 << 30, ldy=1 << 30))])
def test_rows_as_long_as_an_index_are_refused(call, bad):
    assert status(call, ld_codes=1 << 31, ld_scales=1 << 31, **bad) == ac.AC_ERR_INVALID_VALUE


def test_nothing_to_do():
    quantize(rows=0, X=0, codes=0, scales=0)
    quantize(cols=0, ldx=1, ld_codes=1, ld_scales=1, X=0, codes=0, scales=0)
    dequantize(rows=0, codes=0, scales=0, Y=0)
    matmul(M=0, A=0, A_scales=0, Y=0)
    matmul(N=0, B=0, B_scales=0, Y=0, ldy=1)
    gated(F=0, Bg=0, Bu=0, Bg_scales=0, Bu_scales=0, H=0, ldh=1)


def test_workspace_and_kernels():
    for M, N, K in [(1, 4096, 4096), (16, 4096, 14336), (301, 1531, 1001), (4096, 14336, 4096)]:
        for g in (False, True):
            assert ac.adaptcore_mxfp4_kernels(M, N, K, g)
            # the left operand's codes at least, where they are made in a launch of their own
            if len(ac.adaptcore_mxfp4_kernels(M, N, K, g, BF16)) > 1:
                assert ac.adaptcore_mxfp4_workspace(M, N, K, g) >= M * (K // 2)
    assert ac.adaptcore_mxfp4_workspace(0, 5, 5) == 0
    assert ac.adaptcore_mxfp4_kernels(0, 5, 5) == []
    with pytest.raises(ac.AdaptCoreError):
        ac.adaptcore_mxfp4_workspace(-1, 4, 4)
    with pytest.raises(ac.AdaptCoreError):
        ac.adaptcore_mxfp4_kernels(1, 4, 4, False, 9)
