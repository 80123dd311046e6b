"""The feed-forward example: the operators together, trained and served."""
import importlib.util
import os

import pytest

import paper_2608_10803_amd as ac

pytestmark = pytest.mark.gpu


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


def test_trains_and_serves(example):
    block, losses = example.train(steps=40)
    assert losses[-1] < 0.5 * losses[0], losses
    y, ref = example.serve(block)
    # five roundings to bfloat16 on the way (n, H, the adapters' T, Y, the sum
    # with x), each below 2^-8 / sqrt(3) of its value
    assert float((y.double() - ref).norm() / ref.norm()) <= 5 * 2.0 ** -8


def test_gradients_of_the_block(example):
    """The whole block's gradient along random directions against central
    differences of the 64-bit block (the roundings inside: 2^-8 each, of which
    a direction of unit normals sees the norm of the error)."""
    import torch
    b = example.Block(64, 176, seed=5)
    x = torch.randn(50, 64, device="cuda").bfloat16()
    dy = torch.randn(50, 64, device="cuda").bfloat16()
    b.forward(x)
    dx = b.backward(dy)
    at = [x.double()] + [b.master[0].double(), b.master[1].double()] + [m.double() for m in b.matrix]

    def loss(x, w, c, wg, wu, wd):
        n = torch.nn.functional.layer_norm(x, (64,), w, c)
        gate = n @ wg.t()
        return ((x + (gate * torch.sigmoid(gate) * (n @ wu.t())) @ wd.t()) * dy.double()).sum()

    for i, grad in enumerate([dx] + b.grad):
        v = torch.randn(at[i].shape, device="cuda", dtype=torch.float64)
        hi, lo = list(at), list(at)
        hi[i], lo[i] = at[i] + 1e-5 * v, at[i] - 1e-5 * v
        d = (loss(*hi) - loss(*lo)) / 2e-5
        # six roundings on the way, five standard deviations
        assert abs((grad.double() * v).sum() - d) <= 5 * 6 * 2.0 ** -8 * grad.double().norm(), i
