"""What the feed-forward block's entry points refuse, and what they plan (no
GPU)."""
import pytest

import paper_2608_10803_amd as ac

BF16, F16, F32 = ac.AC_TYPE_BF16, ac.AC_TYPE_F16, ac.AC_TYPE_F32
P = 1 << 20  # an aligned address that is never read


def block(**k):
    a = dict(M=4, D=16, F=24, type=BF16, layouts=0, activation=0, X=P, ldx=16, Wg=P, Wu=P, ldw=24, Wd=P, ldd=16, H=P,
             ldh=24, G=P, U=P, ldg=24, Y=P, ldy=16)
    a.update(k)
    return ac.adaptcore_gated_ffn(**a)


def half(**k):
    a = dict(M=4, D=16, F=24, type=BF16, layouts=0, activation=0, X=P, ldx=16, Wg=P, Wu=P, ldw=24, H=P, ldh=24)
    a.update(k)
    return ac.adaptcore_gated_matmul(**a)


def backward(**k):
    a = dict(M=4, D=16, F=24, type=BF16, layouts=0, activation=0, dY=P, lddy=16, X=P, ldx=16, Wg=P, Wu=P, ldw=24, Wd=P,
             ldd=16, G=P, U=P, ldg=24, H=P, ldh=24, dX=P, lddx=16, grad_type=BF16, dWg=P, dWu=P, lddw=24, dWd=P, lddd=16)
    a.update(k)
    return ac.adaptcore_gated_ffn_backward(**a)


SIZES = [dict(M=-1), dict(D=-1), dict(F=-1), dict(M=1 << 31), dict(D=1 << 22), dict(F=1 << 22)]
SHARED = SIZES + [dict(ldx=15), dict(ldw=23), dict(ldh=23), dict(X=P + 1), dict(Wu=P + 1), dict(H=0), dict(X=0),
                  dict(ldx=1 << 23), dict(Wg=0)]


@pytest.mark.parametrize("call,bad", [(c, b) for c in (block, half, backward) for b in SHARED]
                         + [(block, b) for b in (dict(ldd=15), dict(ldy=15), dict(Y=0), dict(Wd=0), dict(Y=P + 1),
                                                 dict(G=0), dict(ldg=23))]
                         + [(half, dict(G=P)), (half, dict(U=P)), (half, dict(layouts=1, ldw=15)),
                            (block, dict(layouts=2, ldd=23))]
                         + [(backward, b) for b in (dict(dWg=0), dict(lddw=23), dict(lddd=15), dict(lddx=15),
                                                    dict(lddy=15), dict(G=0), dict(U=0), dict(dY=0), dict(ldg=23),
                                                    dict(grad_type=F32, dWd=P + 2), dict(dX=P + 1))])
def test_refuses(call, bad):
    with pytest.raises(ac.AdaptCoreError) as e:
        call(**bad)
    assert e.value.status == ac.AC_ERR_INVALID_VALUE


@pytest.mark.parametrize("call,bad", [(c, b) for c in (block, half, backward)
                                      for b in (dict(type=F32), dict(type=9), dict(activation=3), dict(activation=-1),
                                                dict(layouts=4))]
                         + [(half, dict(layouts=2)), (backward, dict(grad_type=F16)), (backward, dict(grad_type=5))])
def test_unsupported(call, bad):
    with pytest.raises(ac.AdaptCoreError) as e:
        call(**bad)
    assert e.value.status == ac.AC_ERR_UNSUPPORTED


def test_nothing_to_do():
    block(M=0, X=0, H=0, G=0, U=0, Y=0)
    half(M=0, X=0, H=0)
    half(F=0, ldw=1, ldh=1, Wg=0, Wu=0, H=0)
    backward(dX=0, dWg=0, dWu=0, dWd=0)
    backward(D=0, lddy=1, ldx=1, ldd=1, lddx=1, lddd=1)


def test_workspace_and_kernels():
    assert ac.adaptcore_gated_ffn_workspace(0, 64, 64) == 0
    for s in ((1, 64, 64), (100, 128, 256), (4096, 4096, 14336)):
        assert ac.adaptcore_gated_ffn_workspace(*s, backward=True) >= 4 * s[0] * s[2]  # dG and dU
        ks = ac.adaptcore_gated_ffn_kernels(*s, backward=True)
        assert ks[0].startswith(("k_dgate<", "k_multi<"))
    assert ac.adaptcore_gated_ffn_kernels(4096, 4096, 14336) == ["k_gated<256, 256>"]
    assert ac.adaptcore_gated_ffn_kernels(1, 4096, 14336)[-1] == "k_gated_sum"
    assert ac.adaptcore_gated_ffn_kernels(1, 512, 1536, layouts=ac.AC_FFN_UP_COL) == ["k_rows<1>"]
    for bad in (lambda: ac.adaptcore_gated_ffn_workspace(-1, 4, 4), lambda: ac.adaptcore_gated_ffn_kernels(1, -1, 4)):
        with pytest.raises(ac.AdaptCoreError):
            bad()


def test_choice_holds_over_sizes():
    """Every size plans something, with as many partitions as blocks at most."""
    for M in (1, 16, 17, 64, 65, 300, 4096, 100000):
        for D in (1, 8, 65, 1000, 8192):
            for F in (1, 40, 512, 14336):
                for k in ac.adaptcore_gated_ffn_kernels(M, D, F, backward=True):
                    if " x" in k:
                        assert 2 <= int(k.split(" x")[1]) <= 64


def test_choices_of_one_and_of_two_segments_of_k():
    """The block's second product of depth 2 F and its dX of two segments of
    depth F have the same sizes, but where F is not a multiple of 64 different
    numbers of k-blocks: neither may take the other's split."""
    for M, D, F in ((128, 128, 96), (300, 64, 32), (2000, 200, 1000)):
        for _ in range(2):
            ac.adaptcore_gated_ffn_workspace(M, D, 2 * F)
            assert ac.adaptcore_gated_ffn_workspace(M, D, F, backward=True) > 0


def test_tall_shallow_projections_stay_fused():
    """Wide outputs of a short K: both projections leave one tile as H, without
    fp32 partials of M F elements."""
    for M, D, F in ((4096, 16, 16384), (4096, 64, 16384), (4096, 128, 16384), (2048, 256, 11008), (150000, 64, 16384),
                    (1000000, 8, 4096)):
        assert ac.adaptcore_gated_ffn_kernels(M, D, F, layouts=3) == ["k_gated<128, 128>"], (M, D, F)
        # zero-padded copies of operands of any alignment (up to 9 columns of H more), and Y's partials
        copies = 2 * (M * (D + 8) + M * (F + 8) + 3 * (F + 8) * (D + 8))
        assert ac.adaptcore_gated_ffn_workspace(M, D, F) <= copies + 64 * 4 * M * (D + 8) + 4096


def test_choices_follow_the_profile():
    """The operators' tiles and splits are priced with the planner's profile,
    and chosen anew when it changes."""
    def chosen():
        return ([ac.adaptcore_gated_ffn_kernels(300, 1024, 2048, backward=True),
                 ac.adaptcore_gated_ffn_kernels(100, 2048, 4096)], ac.adaptcore_adapter_kernels(40, 1024, 4096))

    before = chosen()
    hw = ac.adaptcore_get_hw()
    small = ac.adaptcore_get_hw()
    small.n_cu = 16
    try:
        ac.adaptcore_set_hw(small)
        block, adapters = chosen()
        assert block != before[0] and adapters != before[1]
    finally:
        ac.adaptcore_set_hw(hw)
    assert chosen() == before


def test_widest_block_has_operands_the_tile_can_address():
    """Every operand of the pass, dG and dU among them, lies at a pitch that a
    256-row tile's 32-bit byte offsets reach (checked where the launch is laid
    out)."""
    for M, D, F in ((512, 512, 4194296), (4096, 1024, 2200000), (300, 4194303, 64), (4096, 1024, 4194303)):
        assert ac.adaptcore_gated_ffn_workspace(M, D, F, backward=True) > 4 * M * F
        assert ac.adaptcore_gated_ffn_workspace(M, D, F) >= 0


def test_kernels_of_odd_and_empty_sizes():
    """Few rows on rows of odd length run both products on their own plans;
    what has no elements launches nothing."""
    assert ac.adaptcore_gated_ffn_kernels(17, 100, 77) == ["product", "product", "k_gated_sum"]
    assert ac.adaptcore_gated_ffn_kernels(17, 104, 77) == ["product", "product", "k_gated_sum"]
    assert ac.adaptcore_gated_ffn_kernels(17, 100, 77, layouts=1) == ["k_rows<2>"]
    assert ac.adaptcore_gated_ffn_kernels(0, 64, 64) == ac.adaptcore_gated_ffn_kernels(64, 64, 0) == []
    assert ac.adaptcore_gated_ffn_kernels(64, 0, 64, backward=True) == []
    assert len(ac.adaptcore_gated_ffn_kernels(0, 64, 64, backward=True)) == 1  # the weight gradients, cleared
    assert len(ac.adaptcore_gated_ffn_kernels(64, 64, 0, backward=True)) == 1  # dX, cleared


def test_few_rows_on_the_faster_kernel():
    """Both projections of linear layers, at sizes at which the one kernel or
    the other was measured to be the faster, up to 16 rows and up to 32."""
    for M, D, F in ((16, 512, 1536), (32, 512, 1536), (1, 832, 3008), (4, 1856, 448)):
        assert ac.adaptcore_gated_ffn_kernels(M, D, F, layouts=1)[0].startswith("k_rows"), (M, D, F)
    for M, D, F in ((16, 8192, 2048), (32, 8192, 2048), (32, 4096, 14336), (32, 6848, 2432), (32, 3136, 1920)):
        assert not ac.adaptcore_gated_ffn_kernels(M, D, F, layouts=1)[0].startswith("k_rows"), (M, D, F)


def test_more_tiles_than_a_launch_takes():
    assert ac.adaptcore_gated_ffn_workspace(1 << 28, 64, 64) > 0
    for size in ((1 << 30, 64, 64), ((1 << 31) - 1, 8, 8)):
        with pytest.raises(ac.AdaptCoreError) as e:
            ac.adaptcore_gated_ffn_workspace(*size)
        assert e.value.status == ac.AC_ERR_UNSUPPORTED
