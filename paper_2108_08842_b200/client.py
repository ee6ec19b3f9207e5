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
    fp32 parameter vector.  norm: "none", "rms" or "layer", around every block; drop (the chance of
    a 0) and gate need one.  products: "half" (of the 16-bit type) or "mx4"."""

    def __init__(self, ctx: eden.Context, width: int, hidden: int, blocks: int = 1, act: str = "gelu",
                 dtype: torch.dtype = torch.bfloat16, seed: int = 0, norm: str = "none", drop: float = 0.0, gate: bool = False,
                 products: str = "half"):
        if norm not in ("none", "rms", "layer") or products not in ("half", "mx4"):
            raise ValueError("norm is one of none, rms, layer, products one of half, mx4")
        if norm == "none" and (drop or gate or products != "half"):
            raise ValueError("dropout, a gate and products in 4 bits belong to blocks with norms")
        self.ctx, self.width, self.hidden, self.blocks, self.act, self.dtype = ctx, width, hidden, blocks, act, dtype
        self.norm, self.drop, self.gate, self.products = norm, drop, gate, products
        self.shapes = [s for _ in range(blocks) for s in ((hidden, width), (hidden,), (width, hidden), (width,))]
        # behind them, for each block: the norms' weights, their biases, the gate
        vectors = 0 if norm == "none" else (4 if norm == "layer" else 2) + int(gate)
        self.shapes += [(width,)] * (vectors * blocks)
        self.sizes = [torch.Size(s).numel() for s in self.shapes]
        self.d = sum(self.sizes)
        g = torch.Generator(device="cuda:%d" % ctx.device).manual_seed(seed)
        self.vector = torch.zeros(self.d, device=g.device)
        for p in self.parts(self.vector):
            if p.dim() == 2:
                p.copy_(torch.randn(p.shape, generator=g, device=g.device) * p.shape[1] ** -0.5)
        for b in range(blocks if vectors else 0):
            before, after, gated = self._vectors(self.parts(self.vector), b)
            before[0].fill_(1.0)
            after[0].fill_(1.0)
            if gate:
                gated.fill_(0.5)
        self.load(self.vector)
        self._held: List = []
        self._first = None                                    # with norms: the network's input and its statistics

    def _vectors(self, parts: List[torch.Tensor], b: int):
        """(weight, bias) of the norm before block b and of the one after it, and its gate, out of parts()."""
        each = (len(self.shapes) - 4 * self.blocks) // self.blocks
        v = parts[4 * self.blocks + each * b: 4 * self.blocks + each * (b + 1)]
        bias = (v[2], v[3]) if self.norm == "layer" else (None, None)
        return (v[0], bias[0]), (v[1], bias[1]), v[-1] if self.gate else None

    @staticmethod
    def workspace_bytes(tokens: int, width: int, hidden: int) -> int:
        return max(eden.linear_workspace_bytes(tokens, hidden, width), eden.linear_workspace_bytes(tokens, width, hidden),
                   eden.mx4_workspace_bytes(tokens, hidden, width), eden.mx4_workspace_bytes(tokens, width, hidden),
                   eden.block_workspace_bytes(width))

    def parts(self, vector: torch.Tensor) -> List[torch.Tensor]:
        """Views of W1, b1, W2, b2 of every block in a vector of d values, then the norms' and gates'."""
        return [v.view(s) for v, s in zip(vector.split(self.sizes), self.shapes)]

    def load(self, vector: torch.Tensor):
        """Takes fp32 parameters: the products run on copies in the 16-bit type, or in 4 bits (each rounded once)."""
        self.vector = vector
        parts = self.parts(vector)
        self.work = [p.to(self.dtype) for p in parts]
        if self.norm != "none":
            self._norms = [self._vectors(self.work, b) for b in range(self.blocks)]
        if self.products == "mx4":                            # each by rows and, for the input's gradient, by columns
            self._mx4 = [self.ctx.mx4_quantize_both(p) for p in parts[: 4 * self.blocks] if p.dim() == 2]

    def forward(self, x: torch.Tensor, train: bool = True, seed: int = 0) -> torch.Tensor:
        """x [tokens, width] -> [tokens, width]; train: the checkpoints for `backward` are kept, and
        values are dropped by masks of `seed`."""
        if self.norm != "none":
            return self._forward_joined(x, train, seed)
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

    def _norm(self, b: int, after: bool) -> Optional[eden.Norm]:
        return eden.Norm(*self._norms[b][int(after)], kind=self.norm) if b < self.blocks else None

    def _join(self, b: int, drop: float, seed: int) -> dict:
        """What the join behind block b is called with, forward and backward."""
        return dict(after=self._norm(b, True), before=self._norm(b + 1, False), gate=self._norms[b][2], drop=drop, seed=(seed * self.blocks + b) % 2 ** 64)

    def _forward_joined(self, x: torch.Tensor, train: bool, seed: int) -> torch.Tensor:
        ctx, self._held, self._first, mx4 = self.ctx, [], None, self.products == "mx4"
        if train:
            y, stats = ctx.norm(x, self._norm(0, False), stats=True)
            self._first, self._seed = (ctx.checkpoint_save(x), stats), seed
        else:
            y = ctx.norm(x, self._norm(0, False))
        for b in range(self.blocks):
            w1, b1, w2, b2 = self.work[4 * b: 4 * b + 4]
            join = self._join(b, self.drop if train else 0.0, seed)
            if not train:
                if mx4:
                    h = ctx.mx4_linear(ctx.mx4_linear(y, self._mx4[2 * b][0], b1, act=self.act), self._mx4[2 * b + 1][0], b2)
                else:
                    h = ctx.linear(ctx.linear(y, w1, b1, act=self.act), w2, b2)
                j = ctx.block_join(h, x, **join)
            else:
                if mx4:                                       # the weight gradients' operands are the same values by columns
                    rows, y_held = ctx.mx4_quantize_both(y)
                    a, pre = ctx.mx4_linear(rows, self._mx4[2 * b][0], b1, act=self.act, save="pre")
                    rows, a_held = ctx.mx4_quantize_both(a)
                    h, h_held = ctx.mx4_linear(rows, self._mx4[2 * b + 1][0], b2, save="out")
                else:
                    a, pre = ctx.linear(y, w1, b1, act=self.act, save="pre")
                    y_held, a_held = ctx.checkpoint_save(y), ctx.checkpoint_save(a)
                    h, h_held = ctx.linear(a, w2, b2, save="out")
                j = ctx.block_join(h, x, stats=True, **join)
                x_held = ctx.checkpoint_save(j.x) if b + 1 < self.blocks else None
                self._held.append((y_held, pre, a_held, h_held, x_held, j.after_stats, j.before_stats))
            x, y = j.x, j.y
        return x

    def held_bytes(self, whole: bool = False) -> int:
        """What the blocks' kept activations take; whole: with the network's input, which blocks without norms
        count as the first one's, and the norms' statistics: all that is kept for `backward`."""
        kept = sum(t.numel() for held in self._held for c in held if isinstance(c, tuple) for t in c[:2])
        if whole and self._first:
            x, stats = self._first
            kept += sum(t.numel() for t in x)
            kept += sum(4 * t.numel() for held in [(stats,)] + self._held for t in held if isinstance(t, torch.Tensor))
        return kept

    def backward(self, dy: torch.Tensor, gradient: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
        """The gradient of <dy, forward(x)> with respect to the parameters, as one fp32 vector
        (a row of the matrix that Context.encode takes, say; accumulate: added to it)."""
        ctx = self.ctx
        if gradient is None:
            gradient = torch.empty(self.d, device=dy.device)
        g = self.parts(gradient)
        if self.norm != "none":
            self._backward_joined(dy, g, accumulate)
            return gradient
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

    def _backward_joined(self, dx: torch.Tensor, g: List[torch.Tensor], accumulate: bool):
        ctx, dy, more = self.ctx, None, dict(accumulate=accumulate)
        for b in reversed(range(self.blocks)):
            w1, _, w2, _ = self.work[4 * b: 4 * b + 4]
            g_w1, g_b1, g_w2, g_b2 = g[4 * b: 4 * b + 4]
            y, pre, a, h, x, after_stats, before_stats = self._held[b]
            _, g_after, g_gate = self._vectors(g, b)
            g_before = self._vectors(g, b + 1)[0] if b + 1 < self.blocks else (None, None)
            d = ctx.block_join_backward(dx, dy, h, x, after_stats, before_stats, gate_grad=g_gate, after_weight_grad=g_after[0],
                                        after_bias_grad=g_after[1], before_weight_grad=g_before[0], before_bias_grad=g_before[1],
                                        **self._join(b, self.drop, self._seed), **more)
            dx = d.residual
            ctx.act_backward(d.h, None, out=False, bias_grad=g_b2, **more)
            if self.products == "mx4":
                rows, columns = ctx.mx4_quantize_both(d.h)
                ctx.mx4_linear_weight_grad(columns, a, out=g_w2, **more)
                dz, _ = ctx.mx4_linear_input_grad(rows, self._mx4[2 * b + 1][1], pre=pre, act=self.act, bias_grad=g_b1, dtype=self.dtype, **more)
                rows, columns = ctx.mx4_quantize_both(dz)
                ctx.mx4_linear_weight_grad(columns, y, out=g_w1, **more)
                dy = ctx.mx4_linear_input_grad(rows, self._mx4[2 * b][1], dtype=self.dtype)
            else:
                ctx.linear_weight_grad(d.h, a, out=g_w2, **more)
                dz, _ = ctx.linear_input_grad(d.h, w2, pre=pre, act=self.act, bias_grad=g_b1, **more)
                ctx.linear_weight_grad(dz, y, out=g_w1, **more)
                dy = ctx.linear_input_grad(dz, w1)
        (g_weight, g_bias), _, _ = self._vectors(g, 0)
        x, stats = self._first
        ctx.norm_backward(dy, x, stats, self._norm(0, False), out=False, weight_grad=g_weight, bias_grad=g_bias, **more)


def run(clients: int = 4, rounds: int = 20, bits: float = 1.0, tokens: int = 2048, width: int = 1024, hidden: int = 4096,
        blocks: int = 2, rate: float = 0.6, seed: int = 0, norm: str = "none", drop: float = 0.0, gate: bool = False, products: str = "half",
        say=print) -> List[float]:
    """Rounds of training on a fixed random target function; returns the mean loss of each."""
    extra = 0 if norm == "none" else (4 if norm == "layer" else 2) + int(gate)
    d = blocks * (2 * width * hidden + hidden + width + extra * width)
    need = max(eden.workspace_bytes(d, clients), FeedForward.workspace_bytes(tokens, width, hidden))
    ctx = eden.Context(0, workspace_bytes_=need)
    teacher = FeedForward(ctx, width, hidden, blocks, seed=seed + 1)
    student = FeedForward(ctx, width, hidden, blocks, seed=seed + 2, norm=norm, drop=drop, gate=gate, products=products)
    assert student.d == d
    gradients = torch.empty((clients, d), device=student.vector.device)
    losses = []
    for r in range(rounds):
        total = 0.0
        for c in range(clients):
            g = torch.Generator(device=gradients.device).manual_seed(seed * 1000003 + r * clients + c)
            x = torch.randn((tokens, width), generator=g, device=gradients.device).to(student.dtype)
            off = student.forward(x, seed=seed * 1000003 + r * clients + c).float() - teacher.forward(x, train=False).float()
            total += off.square().mean()
            student.backward((off * (2.0 / tokens)).to(student.dtype), gradients[c])
        seeds = [(seed + 1) * 2 ** 40 + r * clients + c + 1 for c in range(clients)]
        codes, scales = ctx.encode(gradients, [bits] * clients, seeds)
        mean = ctx.mean(codes, scales, [bits] * clients, seeds, d)
        student.load(student.vector - rate / width * mean)
        losses.append(float(total) / clients)
        say("round %d: loss %.5f  (%d clients, d = %d, %.3g bits; held activations %.1f MB a client)" % (
            r, losses[-1], clients, d, bits, student.held_bytes(whole=True) / 1e6))
    assert ctx.status() == 0
    ctx.close()
    return losses


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, kind, default in (("clients", int, 4), ("rounds", int, 20), ("bits", float, 1.0), ("tokens", int, 2048), ("width", int, 1024),
                                ("hidden", int, 4096), ("blocks", int, 2), ("rate", float, 0.6), ("seed", int, 0)):
        p.add_argument("--" + name, type=kind, default=default)
    p.add_argument("--norm", choices=("none", "rms", "layer"), default="none")
    p.add_argument("--drop", type=float, default=0.0)
    p.add_argument("--gate", action="store_true")
    p.add_argument("--products", choices=("half", "mx4"), default="half")
    run(**vars(p.parse_args()))


if __name__ == "__main__":
    main()
