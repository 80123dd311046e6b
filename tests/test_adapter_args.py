"""What the adapters' entry point refuses, and what it plans (no GPU)."""
import pytest

import paper_2608_10803_amd as ac

P = 1 << 20  # an aligned address that is never read


def call(**k):
    a = dict(M=4, N=24, K=16, dtype=ac.AC_BF16_BF16OUT, layouts=0, X=P, ldx=16, W=P, ldw=24, adapters=3, rank=8, down=P,
             ld_down=16, stride_down=128, up=P, ld_up=8, stride_up=192, index=P, scale=P, bias=P, Y=P, ldy=24)
    a.update(k)
    return ac.adaptcore_adapter_matmul(**a)


@pytest.mark.parametrize("bad", [dict(M=-1), dict(N=-1), dict(K=-1), dict(M=1 << 22), dict(N=1 << 22), dict(K=1 << 22),
                                 dict(adapters=-1), dict(adapters=1 << 31), dict(rank=-1), dict(rank=4097), dict(ldx=15),
                                 dict(ldw=23), dict(layouts=2, ldw=15), dict(ldy=23), dict(ld_down=15), dict(ld_up=7),
                                 dict(stride_down=-1), dict(stride_up=-1), dict(stride_up=1 << 40), dict(X=0), dict(W=0),
                                 dict(Y=0), dict(down=0), dict(up=0), dict(index=0), dict(X=P + 1), dict(W=P + 1),
                                 dict(down=P + 1), dict(up=P + 1), dict(Y=P + 1), dict(index=P + 2), dict(scale=P + 2),
                                 dict(bias=P + 1), dict(dtype=ac.AC_BF16_F32OUT, Y=P + 2), dict(ldx=1 << 23)])
def test_refuses(bad):
    with pytest.raises(ac.AdaptCoreError) as e:
        call(**bad)
    assert e.value.status == ac.AC_ERR_INVALID_VALUE


@pytest.mark.parametrize("bad", [dict(dtype=4), dict(dtype=-1), dict(layouts=1), dict(layouts=4)])
def test_unsupported(bad):
    with pytest.raises(ac.AdaptCoreError) as e:
        call(**bad)
    assert e.value.status == ac.AC_ERR_UNSUPPORTED


def test_nothing_to_do():
    call(M=0, X=0, Y=0, index=0)
    call(N=0, ldw=1, W=0, Y=0, up=0)


def test_workspace_and_kernels():
    assert ac.adaptcore_adapter_workspace(0, 64, 64, 4) == 0
    for s in ((1, 64, 64, 4), (64, 14336, 4096, 64), (4096, 4096, 4096, 16), (77, 333, 1001, 5)):
        assert ac.adaptcore_adapter_workspace(*s) >= 2 * s[0] * s[3]
    assert ac.adaptcore_adapter_kernels(4096, 14336, 4096) == ["k_shrink", "k_adapter<256, 256>"]
    assert ac.adaptcore_adapter_kernels(1, 4096, 4096)[-1] == "k_adapter_sum"
    for bad in (lambda: ac.adaptcore_adapter_workspace(-1, 4, 4, 4), lambda: ac.adaptcore_adapter_kernels(1, -1, 4)):
        with pytest.raises(ac.AdaptCoreError):
            bad()


def test_kernels_of_a_call():
    """T beside the partial sums up to 64 rows and rank 64, in a launch of its
    own past either, and none without adapters."""
    for rank, first in ((1, ["k_multi_shrink<32, 128> x5"]), (64, ["k_multi_shrink<32, 128> x5"]),
                        (65, ["k_shrink", "k_multi<32, 128> x5"]), (0, ["k_multi<32, 128> x5"])):
        assert ac.adaptcore_adapter_kernels(16, 4096, 4096, rank) == first + ["k_adapter_sum"]
    assert ac.adaptcore_adapter_kernels(16, 4096, 4096, 16, adapters=0) == ["k_multi<32, 128> x5", "k_adapter_sum"]
    assert ac.adaptcore_adapter_kernels(300, 512, 4096, 16) == ["k_shrink", "k_multi<32, 128> x5", "k_adapter_sum"]
    assert ac.adaptcore_adapter_kernels(4096, 14336, 4096, 16) == ac.adaptcore_adapter_kernels(4096, 14336, 4096)
    assert ac.adaptcore_adapter_kernels(0, 64, 64, 4) == ac.adaptcore_adapter_kernels(64, 0, 64, 4) == []
    for bad in ((1, 4, 4, -1), (1, 4, 4, 4097), (-1, 4, 4, 4)):
        with pytest.raises(ac.AdaptCoreError):
            ac.adaptcore_adapter_kernels(*bad)
    with pytest.raises(ac.AdaptCoreError):
        ac.adaptcore_adapter_kernels(1, 4, 4, 4, adapters=-1)
