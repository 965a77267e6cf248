"""Adapters of several requests beside shared 4-bit weights: fine-tuned from 8-bit checkpoints, then served.

A stack of residual blocks, each a projection whose weight is frozen in packed piecewise linear codes:

    x, codes, step = norm_block(x + gate * norm(f))      the norms around the last block, its output in 8 bits
    y              = linear_i8(codes, packed weight)     one integer product for all requests, in units of a row's step
    f, h           = adapter(codes, base=y)              plus what each row's own adapter adds

The weights cannot learn; adapters, norms and gates do.  A training step keeps for its backward pass the codes that the
product took anyway, the ranks h, and the residual stream and block outputs in 8 bits.  Serving runs the same calls on
prompts and on one token of each request.

    python examples/adapters_beside_packed_weights.py [--width 1024] [--blocks 4] [--rank 16] [--adapters 4] [--steps 20]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2002_00104_amd import block, pwlq  # noqa: E402

BITS = 4
EPS = 1e-6


class Projection:
    """A frozen [N, K] weight in packed codes, and the rounded weight that the gradient of its input takes."""

    def __init__(self, weight):
        found = pwlq.search(weight, BITS, 200, fast=True)
        self.p, self.m, self.rows = found["p_star"], found["m"], weight.shape[0]
        self.codes, self.flags, w_hat = pwlq.quantize_packed(weight, BITS, self.p, self.m)
        self.w_hat = w_hat.to(torch.bfloat16)

    def __call__(self, codes):
        """In units of a row's step: activations have one for each row, which the adapters' epilogue multiplies with."""
        return pwlq.linear_i8(codes, 1.0, 0.0, self.codes, self.flags, self.rows, BITS, self.p, self.m)[0]


class Block:
    """Norms, gate, projection and the adapters [n, R, width] of one block, all but the projection trainable."""

    def __init__(self, width, rank, adapters, first, generator):
        def normal(*shape, scale):
            return torch.randn(shape, generator=generator, device="cuda") * scale

        self.projection = Projection(normal(width, width, scale=width ** -0.5))
        self.first = first                                     # the first block's input is no block's output
        self.master = dict(pre=torch.ones(width, device="cuda"), down=normal(adapters, rank, width, scale=width ** -0.5),
                           up=torch.zeros(adapters, rank, width, device="cuda"))
        if not first:
            self.master.update(post=torch.ones(width, device="cuda"), gate=torch.full((1, width), 0.5, device="cuda"))
        self.scale = torch.ones(adapters, device="cuda")
        self.cast()

    def cast(self):
        """The 16-bit copies that the kernels read, from the trained binary32 parameters."""
        self.down, self.up = (self.master[k].to(torch.bfloat16) for k in ("down", "up"))
        self.norms = dict(pre_weight=self.master["pre"], eps=EPS)
        if not self.first:
            self.norms.update(post_weight=self.master["post"], gate=self.master["gate"].to(torch.bfloat16))


class Stack:
    def __init__(self, width=1024, blocks=4, rank=16, adapters=4, seed=0):
        generator = torch.Generator(device="cuda").manual_seed(seed)
        self.blocks = [Block(width, rank, adapters, i == 0, generator) for i in range(blocks)]
        self.pre = torch.ones(width, device="cuda")

    def forward(self, x, ids, keep=None):
        """x [T, width] bfloat16, ids int32 [T] (-1: no adapter).  `keep`: a list that receives the checkpoints."""
        f = None
        for b in self.blocks:
            x, codes, step = block.norm_block(x, f, pack=True, **b.norms)
            y, h = block.adapter(codes, b.down, b.up, ids, b.scale, base=b.projection(codes), x_step=step, base_step=step)
            if keep is not None:
                keep.append((block.pack_rows(x), None if f is None else block.pack_rows(f), codes, step, h))
            f = y
        x, u = block.norm_block(x, f, pre_weight=self.pre, eps=EPS)
        if keep is not None:
            keep.append((block.pack_rows(x), block.pack_rows(f)))
        return u

    def backward(self, du, ids, kept):
        """Gradients of every block's parameters from that of the output, du bfloat16; of rounding to 8 bits, the identity's."""
        (x, x_step), (f, f_step) = kept[-1]
        got = block.norm_block_backward(du, None, x, f, pre_weight=self.pre, eps=EPS, x_step=x_step, f_step=f_step)
        gradients = []
        for b, ((x, x_step), output, codes, step, h) in zip(self.blocks[::-1], kept[-2::-1]):
            dx, dy = got["dx"], got["df"]
            low = block.adapter_backward(dy, codes, b.down, b.up, ids, b.scale, h, x_step=step, dx_base=dy @ b.projection.w_hat)
            if output is None:                                 # the norm alone: its input is the residual stream as it was kept
                f, f_step = None, None
            else:
                f, f_step = output
            got = block.norm_block_backward(low["dx"], dx, x, f, x_step=x_step, f_step=f_step, **b.norms)
            gradients.append({k: v for k, v in dict(down=low["d_down"], up=low["d_up"], pre=got["d_pre"], post=got["d_post"],
                                                    gate=got["d_gate"]).items() if k in b.master})
        return gradients[::-1]

    def parameters(self):
        return [p for b in self.blocks for p in b.master.values()]

    def step(self, x, ids, target, optimizer):
        """One step on half the squared error of a row; returns that of a mean row before it."""
        kept = []
        off = self.forward(x, ids, kept).float() - target
        for b, g in zip(self.blocks, self.backward((off / x.shape[0]).to(torch.bfloat16), ids, kept)):
            for name, parameter in b.master.items():
                parameter.grad = g[name]
        optimizer.step()
        for b in self.blocks:
            b.cast()
        return 0.5 * off.square().sum(1).mean()


def main():
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in dict(width=1024, blocks=4, rank=16, adapters=4, steps=20, rows=512).items():
        parser.add_argument("--" + name, type=int, default=default)
    parser.add_argument("--rate", type=float, default=5e-3)
    a = parser.parse_args()
    stack = Stack(a.width, a.blocks, a.rank, a.adapters)
    generator = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((a.rows, a.width), generator=generator, device="cuda").to(torch.bfloat16)
    # prompts of one request after the other, the first rows without an adapter
    ids = (torch.arange(a.rows, device="cuda", dtype=torch.int32) * (a.adapters + 1)).div(a.rows, rounding_mode="floor").to(torch.int32) - 1
    # each adapter learns a fixed change of the output of its own
    change = torch.randn((a.adapters + 1, a.width), generator=generator, device="cuda")
    change[0] = 0.0
    target = stack.forward(x, ids).float() + 0.5 * change[ids.long() + 1]
    optimizer = torch.optim.Adam(stack.parameters(), lr=a.rate)
    for i in range(a.steps):
        loss = stack.step(x, ids, target, optimizer)
        if i % 5 == 0 or i == a.steps - 1:
            print(f"step {i}: loss {loss.item():.1f}", flush=True)
    # a batch that decodes: one token of each adapter and one without
    last = torch.tensor([int((ids == k).nonzero()[-1]) for k in range(-1, a.adapters)], device="cuda")
    served = stack.forward(x[last].contiguous(), ids[last].contiguous())
    print(f"served one token of {len(last)} requests, loss {0.5 * (served.float() - target[last]).square().sum(1).mean().item():.1f}")


if __name__ == "__main__":
    main()
