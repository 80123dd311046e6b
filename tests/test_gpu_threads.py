"""Calls of two host threads on one stream: every call's launches share the
stream's workspace, so each call is enqueued whole. The same calls one after the
other give the expected bits."""
import threading

import pytest

import paper_2608_10803_amd as ac

pytestmark = pytest.mark.gpu

CALLS = 60


@pytest.fixture(scope="module")
def t():
    import torch
    assert torch.cuda.is_available()
    ac.adaptcore_init()
    return torch


def norm_backward(t, g):
    x, dy = (t.randn(600, 2000, device="cuda", generator=g) for _ in range(2))
    m, r, dx = x.mean(1), x.std(1).reciprocal(), t.empty_like(x)

    def call(out, stream):
        ac.layer_norm_backward_tensors(dy, x, None, m, r, dx, dweight=out[0], dbias=out[1], stream=stream)

    return call, lambda: t.empty(2, 2000, device="cuda")


def split_product(t, g):
    a, b = (t.randn(s, device="cuda", generator=g).bfloat16() for s in ((96, 20000), (20000, 80)))
    assert ac.adaptcore_plan_info(ac.adaptcore_plan(96, 80, 20000, ac.AC_BF16_F32OUT)).get("workspace_bytes") > 0
    return (lambda out, stream: ac.matmul_tensors(a, b, out, stream=stream)), lambda: t.empty(96, 80, device="cuda")


def block(t, g):
    x, wg, wu, wd = (t.randn(s, device="cuda", generator=g).bfloat16() for s in ((70, 101), (101, 333), (101, 333),
                                                                                  (333, 101)))
    h = t.empty(70, 333, device="cuda", dtype=t.bfloat16)

    def call(out, stream):
        ac.gated_ffn_tensors(x, wg, wu, wd, h, out, stream=stream)

    return call, lambda: t.empty(70, 101, device="cuda", dtype=t.bfloat16)


def adapters(t, g):
    x, w = t.randn(40, 1024, device="cuda", generator=g).bfloat16(), t.randn(1024, 512, device="cuda", generator=g).bfloat16()
    down, up = (t.randn(s, device="cuda", generator=g).bfloat16() for s in ((4, 16, 1024), (4, 512, 16)))
    index = t.randint(-1, 4, (40,), device="cuda", generator=g, dtype=t.int32)

    def call(out, stream):
        ac.adapter_mm_tensors(x, w, down, up, index, out, stream=stream)

    return call, lambda: t.empty(40, 512, device="cuda", dtype=t.bfloat16)


@pytest.mark.parametrize("which", ["stream", "per_thread"])
@pytest.mark.parametrize("make", [norm_backward, split_product, block, adapters], ids=lambda f: f.__name__)
def test_two_threads(t, make, which):
    stream = t.cuda.Stream()
    handle = stream.cuda_stream if which == "stream" else 2  # (hipStreamPerThread)
    jobs = []
    for seed in (1, 2):
        call, empty = make(t, t.Generator(device="cuda").manual_seed(seed))
        ref = empty()
        t.cuda.synchronize()
        call(ref, stream.cuda_stream)
        jobs.append((call, ref, [empty() for _ in range(CALLS)]))
    t.cuda.synchronize()
    start, errors = threading.Barrier(2), []

    def work(call, outs):
        try:
            t.cuda.set_device(0)
            start.wait()
            for out in outs:
                call(out, handle)
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(call, outs)) for call, _, outs in jobs]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    t.cuda.synchronize()
    assert not errors, errors
    for _, ref, outs in jobs:
        assert all(t.equal(out, ref) for out in outs)
