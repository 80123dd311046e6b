"""A transformer's feed-forward block on the library's operators, trained and
served:

    y = x + (act(n Wg) * (n Wu)) Wd,   n = layer norm of x

Training: layer_norm_tensors and gated_ffn_tensors forward,
gated_ffn_backward_tensors (32-bit weight gradients) and
layer_norm_backward_tensors backward, plain gradient descent on 32-bit master
weights; the block learns a fixed random one from its outputs.

Serving: the trained block's down-projection is shared by requests that each
bring a low-rank adapter of it: gated_mm_tensors, then adapter_mm_tensors for
all of them at once, prompts and single tokens in one batch.

    python examples/feed_forward_block.py [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_10803_amd as ac  # noqa: E402


class Block:
    """The block's weights (32-bit masters, and the bfloat16 matrices the
    products read, stored as a linear layer's) and its calls."""

    def __init__(self, dim, hidden, seed, act="silu"):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(out, inp):
            return torch.randn(out, inp, device="cuda", generator=g) * inp ** -0.5

        self.act, self.dim, self.hidden = act, dim, hidden
        self.master = [torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda"), weight(hidden, dim),
                       weight(hidden, dim), weight(dim, hidden)]
        self.grad = [torch.empty_like(m) for m in self.master]
        self.matrix = [m.bfloat16() for m in self.master[2:]]

    def views(self, of):
        """Wg, Wu (dim x hidden) and Wd (hidden x dim) as the products take them."""
        return [m.t() for m in of]

    def norm(self, x):
        n = torch.empty_like(x)
        mean, rstd = (torch.empty(x.shape[0], device="cuda") for _ in range(2))
        ac.layer_norm_tensors(x, self.master[0], self.master[1], n, mean=mean, rstd=rstd)
        return n, mean, rstd

    def forward(self, x):
        n, mean, rstd = self.norm(x)
        h, gate, up = (torch.empty(x.shape[0], self.hidden, device="cuda", dtype=x.dtype) for _ in range(3))
        y = torch.empty_like(x)
        ac.gated_ffn_tensors(n, *self.views(self.matrix), h, y, act=self.act, gate=gate, up=up)
        self.saved = x, n, mean, rstd, gate, up, h
        return y.add_(x)

    def backward(self, dy):
        x, n, mean, rstd, gate, up, h = self.saved
        dn, dx = torch.empty_like(x), torch.empty_like(x)
        dwg, dwu, dwd = self.views(self.grad[2:])
        ac.gated_ffn_backward_tensors(dy, n, *self.views(self.matrix), gate, up, h, dX=dn, dWg=dwg, dWu=dwu, dWd=dwd,
                                      act=self.act)
        ac.layer_norm_backward_tensors(dn, x, self.master[0], mean, rstd, dx, dweight=self.grad[0], dbias=self.grad[1])
        return dx.add_(dy)

    def step(self, rate):
        for m, g in zip(self.master, self.grad):
            m.sub_(g, alpha=rate)
        for b, m in zip(self.matrix, self.master[2:]):
            b.copy_(m)

    def serve(self, x, down, up, index, scale):
        """The block for rows of many requests, each with its adapter of the
        down-projection."""
        n, _, _ = self.norm(x)
        h = torch.empty(x.shape[0], self.hidden, device="cuda", dtype=x.dtype)
        y = torch.empty_like(x)
        wg, wu, wd = self.views(self.matrix)
        ac.gated_mm_tensors(n, wg, wu, h, act=self.act)
        ac.adapter_mm_tensors(h, wd, down, up, index, y, scale=scale)
        return y.add_(x)


def train(dim=256, hidden=704, tokens=1000, steps=60, rate=0.5):
    """Losses of a block that learns another one's outputs."""
    teacher, block = Block(dim, hidden, seed=1), Block(dim, hidden, seed=2)
    g = torch.Generator(device="cuda").manual_seed(3)
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, dim, device="cuda", generator=g).bfloat16()
        with torch.no_grad():
            e = block.forward(x).float() - teacher.forward(x).float()
        losses.append(e.pow(2).mean())
        block.backward((e * (2.0 / tokens)).bfloat16())
        block.step(rate)
    return block, [float(v) for v in losses]


def serve(block, adapters=5, rank=12, prompts=(300, 41), singles=20):
    """Outputs of a mixed batch and, for comparison, the same in 64 bits with
    each request's adapter merged into the weight."""
    g = torch.Generator(device="cuda").manual_seed(4)

    def values(*shape, scale=1.0):
        return (torch.randn(*shape, device="cuda", generator=g) * scale).bfloat16()

    lengths = list(prompts) + [1] * singles
    which = torch.randint(-1, adapters, (len(lengths),), device="cuda", generator=g)
    index = torch.repeat_interleave(which, torch.tensor(lengths, device="cuda")).int()
    x = values(index.numel(), block.dim)
    down = values(adapters, rank, block.hidden, scale=block.hidden ** -0.5)
    up = values(adapters, block.dim, rank, scale=rank ** -0.5)
    scale = torch.linspace(0.5, 1.5, adapters, device="cuda")
    y = block.serve(x, down, up, index, scale)

    n = torch.nn.functional.layer_norm(x.double(), (block.dim,), block.master[0].double(), block.master[1].double())
    wg, wu, wd = (m.double().t() for m in block.matrix)
    gate = n @ wg
    h = gate * torch.sigmoid(gate) * (n @ wu)
    ref = x.double() + h @ wd
    for a in range(adapters):
        rows = index == a
        ref[rows] += scale[a].double() * (h[rows] @ down[a].double().t()) @ up[a].double().t()
    return y, ref


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    block, losses = train(steps=ap.parse_args().steps)
    for i in range(0, len(losses), 10):
        print("step %3d  loss %.4f" % (i, losses[i]))
    print("step %3d  loss %.4f" % (len(losses) - 1, losses[-1]))
    y, ref = serve(block)
    print("served %d rows: relative error %.2g against 64 bits"
          % (y.shape[0], float((y.double() - ref).norm() / ref.norm())))


if __name__ == "__main__":
    main()
