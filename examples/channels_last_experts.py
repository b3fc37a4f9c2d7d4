"""A residual block of a channels-last network whose pointwise layers are a mixture of experts, in 8-bit floats:

    group norm + SiLU -> codes                      (one call: the norm leaves the products' operand)
    codes x router                                  product in blocks, 32-bit scores
    two experts a position, rows sorted by expert
    codes x first layer of the experts, SiLU        rows picked from the positions by an index
    -> codes, x second layer of the experts         quantised, grouped again
    + x                                             32-bit rows back to their positions, weighted with the scores; rounded once

    python examples/channels_last_experts.py [samples] [height] [width] [channels]

Prints how far the block is from the same formulas in 32 bits on the unquantised weights, and its time.
"""
from __future__ import annotations

import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2112_15445_amd import binding as B  # noqa: E402


class Block:
    """Weights of a block of C channels with E experts of `hidden` channels: kept in 32 bits for the comparison, used as codes."""

    def __init__(self, C, E=8, hidden=None, groups=32, top=2, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        hidden = 2 * C if hidden is None else hidden
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.groups, self.top = groups, top
        self.gamma, self.beta = 1 + 0.1 * rand(C), 0.1 * rand(C)
        self.router, self.first, self.second = rand(E, C) * C ** -0.5, rand(E, hidden, C) * C ** -0.5, rand(E, C, hidden) * hidden ** -0.5
        self.bias = 0.1 * rand(E, hidden)
        # (once, when the model is loaded)
        self.router_q, self.first_q, self.second_q = (B.quantize_blocks_torch(w, 128) for w in (self.router, self.first, self.second))

    def forward(self, x):
        """x [N, S, C] in 16 bits."""
        q, scale = B.group_norm_torch(x, self.groups, self.gamma, self.beta, act="silu", codes=True)
        scores = B.matmul_blocks_torch(q, scale, *self.router_q, dtype=torch.float32)
        ids, weights = B.route_experts_torch(scores, self.top)
        offsets, index, position = B.sort_by_expert_torch(ids, self.first.shape[0])
        h = B.matmul_grouped_torch(q, self.first_q[0], offsets, scale, self.first_q[1], index=index, bias=self.bias, act="silu")
        hq, h_scale = B.quantize_blocks_torch(h)
        y = B.matmul_grouped_torch(hq, self.second_q[0], offsets, h_scale, self.second_q[1], dtype=torch.float32)
        out = B.combine_rows_torch(y, position, weights, residual=x.view(-1, x.shape[-1]).float())
        return out.view(x.shape).to(x.dtype), (weights, offsets, index, position)

    def reference(self, x, chosen):
        """The same in 32 bits, with the experts that were chosen."""
        weights, offsets, index, position = chosen
        N, S, C = x.shape
        z = torch.nn.functional.group_norm(x.float().transpose(1, 2), self.groups, self.gamma, self.beta).transpose(1, 2)
        z = torch.nn.functional.silu(z).reshape(N * S, C)
        rows, bounds = z[index.long()], offsets.tolist()
        y = torch.cat([torch.nn.functional.silu(rows[lo:hi] @ w.t() + b) @ v.t()
                       for lo, hi, w, b, v in zip(bounds, bounds[1:], self.first, self.bias, self.second)])
        return x.float() + (y[position.long()] * weights[:, :, None]).sum(1).view(x.shape)


def main(N=8, H=28, W=28, C=512):
    block = Block(C)
    x = torch.randn(N, H * W, C, device="cuda").to(torch.bfloat16)
    y, chosen = block.forward(x)
    ref = block.reference(x, chosen)
    added, wanted = y.float() - x.float(), ref - x.float()
    off = float((added - wanted).norm() / wanted.norm())
    for _ in range(3):
        block.forward(x)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(20):
        block.forward(x)
    torch.cuda.synchronize()
    print(f"{N} x {H}x{W} x {C}, {block.first.shape[0]} experts: what the block adds is {off:.3f} off the 32-bit formulas; "
          f"{(time.perf_counter() - t) / 20 * 1e6:.0f} us a pass")
    return off


if __name__ == "__main__":
    sys.exit(0 if main(*(int(v) for v in sys.argv[1:])) < 0.1 else 1)
