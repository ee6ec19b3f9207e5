"""A sender that trains: feed-forward blocks whose activations are kept in 8 bits and whose
gradient is the vector that EDEN sends.

    y = x + W2 act(W1 x + b1) + b2          for each block, tokens as rows

The parameters of all blocks are one fp32 vector, as is the gradient: ``backward`` writes every
weight and bias gradient into its place in the vector that ``Context.encode`` takes, so nothing
is gathered or copied between the backward pass and the sender.  Between the passes a block
holds its input, its pre-activation and its hidden activations as 8-bit checkpoints.

    python -m paper_2108_08842_b200.client --clients 4 --rounds 20 --bits 1

runs rounds of distributed mean estimation on one GPU: each client computes its gradient on its
own batch, encodes it, the receiver estimates the mean of all clients' vectors and every client
takes the same step.
"""
from __future__ import annotations

import argparse
from typing import List, Optional

import torch

from . import eden


class FeedForward:
    """`blocks` residual blocks of `width` features with `hidden` units, bf16 or fp16 over an
    fp32 parameter vector."""

    def __init__(self, ctx: eden.Context, width: int, hidden: int, blocks: int = 1, act: str = "gelu",
                 dtype: torch.dtype = torch.bfloat16, seed: int = 0):
        self.ctx, self.width, self.hidden, self.blocks, self.act, self.dtype = ctx, width, hidden, blocks, act, dtype
        self.shapes = [s for _ in range(blocks) for s in ((hidden, width), (hidden,), (width, hidden), (width,))]
        self.sizes = [torch.Size(s).numel() for s in self.shapes]
        self.d = sum(self.sizes)
        g = torch.Generator(device="cuda:%d" % ctx.device).manual_seed(seed)
        self.vector = torch.zeros(self.d, device=g.device)
        for p in self.parts(self.vector):
            if p.dim() == 2:
                p.copy_(torch.randn(p.shape, generator=g, device=g.device) * p.shape[1] ** -0.5)
        self.load(self.vector)
        self._held: List = []

    @staticmethod
    def workspace_bytes(tokens: int, width: int, hidden: int) -> int:
        return max(eden.linear_workspace_bytes(tokens, hidden, width), eden.linear_workspace_bytes(tokens, width, hidden))

    def parts(self, vector: torch.Tensor) -> List[torch.Tensor]:
        """Views of W1, b1, W2, b2 of every block in a vector of d values."""
        return [v.view(s) for v, s in zip(vector.split(self.sizes), self.shapes)]

    def load(self, vector: torch.Tensor):
        """Takes fp32 parameters: the products run on copies in the 16-bit type."""
        self.vector = vector
        self.work = [p.to(self.dtype) for p in self.parts(vector)]

    def forward(self, x: torch.Tensor, train: bool = True) -> torch.Tensor:
        """x [tokens, width] -> [tokens, width]; train: the checkpoints for `backward` are kept."""
        ctx, self._held = self.ctx, []
        saved = ctx.checkpoint_save(x) if train else None
        for b in range(self.blocks):
            w1, b1, w2, b2 = self.work[4 * b: 4 * b + 4]
            if not train:
                x = ctx.linear(ctx.linear(x, w1, b1, act=self.act), w2, b2, residual=x)
                continue
            h, pre = ctx.linear(x, w1, b1, act=self.act, save="pre")
            x, after = ctx.linear(h, w2, b2, residual=x, save="out")
            self._held.append((saved, pre, ctx.checkpoint_save(h)))
            saved = after                                     # the next block's input
        return x

    def held_bytes(self) -> int:
        """What the kept activations take."""
        return sum(t.numel() for held in self._held for c in held for t in c)

    def backward(self, dy: torch.Tensor, gradient: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
        """The gradient of <dy, forward(x)> with respect to the parameters, as one fp32 vector
        (a row of the matrix that Context.encode takes, say; accumulate: added to it)."""
        ctx = self.ctx
        if gradient is None:
            gradient = torch.empty(self.d, device=dy.device)
        g = self.parts(gradient)
        ctx.act_backward(dy, None, out=False, bias_grad=g[-1], accumulate=accumulate)
        for b in reversed(range(self.blocks)):
            w1, _, w2, _ = self.work[4 * b: 4 * b + 4]
            g_w1, g_b1, g_w2, _ = g[4 * b: 4 * b + 4]
            x, pre, h = self._held[b]
            ctx.linear_weight_grad(dy, h, out=g_w2, accumulate=accumulate)
            dz, _ = ctx.linear_input_grad(dy, w2, pre=pre, act=self.act, bias_grad=g_b1, accumulate=accumulate)
            ctx.linear_weight_grad(dz, x, out=g_w1, accumulate=accumulate)
            if b > 0:                                         # its sums are the gradient of the block below's b2
                dy, _ = ctx.linear_input_grad(dz, w1, residual=dy, bias_grad=g[4 * b - 1], accumulate=accumulate)
        return gradient


def run(clients: int = 4, rounds: int = 20, bits: float = 1.0, tokens: int = 2048, width: int = 1024, hidden: int = 4096,
        blocks: int = 2, rate: float = 0.6, seed: int = 0, say=print) -> List[float]:
    """Rounds of training on a fixed random target function; returns the mean loss of each."""
    d = blocks * (2 * width * hidden + hidden + width)
    need = max(eden.workspace_bytes(d, clients), FeedForward.workspace_bytes(tokens, width, hidden))
    ctx = eden.Context(0, workspace_bytes_=need)
    teacher = FeedForward(ctx, width, hidden, blocks, seed=seed + 1)
    student = FeedForward(ctx, width, hidden, blocks, seed=seed + 2)
    assert student.d == d
    gradients = torch.empty((clients, d), device=student.vector.device)
    losses = []
    for r in range(rounds):
        total = 0.0
        for c in range(clients):
            g = torch.Generator(device=gradients.device).manual_seed(seed * 1000003 + r * clients + c)
            x = torch.randn((tokens, width), generator=g, device=gradients.device).to(student.dtype)
            off = student.forward(x).float() - teacher.forward(x, train=False).float()
            total += off.square().mean()
            student.backward((off * (2.0 / tokens)).to(student.dtype), gradients[c])
        seeds = [(seed + 1) * 2 ** 40 + r * clients + c + 1 for c in range(clients)]
        codes, scales = ctx.encode(gradients, [bits] * clients, seeds)
        mean = ctx.mean(codes, scales, [bits] * clients, seeds, d)
        student.load(student.vector - rate / width * mean)
        losses.append(float(total) / clients)
        say("round %d: loss %.5f  (%d clients, d = %d, %.3g bits; held activations %.1f MB a client)" % (
            r, losses[-1], clients, d, bits, student.held_bytes() / 1e6))
    assert ctx.status() == 0
    ctx.close()
    return losses


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, kind, default in (("clients", int, 4), ("rounds", int, 20), ("bits", float, 1.0), ("tokens", int, 2048), ("width", int, 1024),
                                ("hidden", int, 4096), ("blocks", int, 2), ("rate", float, 0.6), ("seed", int, 0)):
        p.add_argument("--" + name, type=kind, default=default)
    run(**vars(p.parse_args()))


if __name__ == "__main__":
    main()
