"""A small stack of feed-forward blocks trained and served in 8 bits.

Everything that the blocks save between their forward and backward passes is held in 8 bits (FeedForward8), everything
that the optimizer holds between steps at the widths of its policy (STQAdamW).  Afterwards the weights are frozen in 8
bits and one token at a time goes through the same blocks.

    python examples/feed_forward_8bit.py [--steps 60] [--width 256] [--hidden 704] [--blocks 2]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_06836_b200.ffn8 import FeedForward8  # noqa: E402
from paper_2604_06836_b200.optim import STQAdamW  # noqa: E402


class Stack(torch.nn.Module):
    def __init__(self, width, hidden, blocks, kind="silu_gated"):
        super().__init__()
        self.blocks = torch.nn.ModuleList(FeedForward8(width, hidden, kind) for _ in range(blocks))

    def forward(self, x):
        h = None
        for b in self.blocks:
            x, h = b(x, h)
        return x + h


def train(model, steps, width, tokens=512, seed=0, lr=2e-3):
    """Learns a fixed random map of unit rows; returns the losses."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    target = torch.randn(width, width, device="cuda", generator=gen) / width ** 0.5
    opt = STQAdamW(model.parameters(), lr=lr, weight_decay=0.0, policy="paper", interval=10)
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, width, device="cuda", generator=gen)
        opt.zero_grad()
        loss = torch.nn.functional.mse_loss(model(x.bfloat16()).float(), torch.tanh(x @ target))
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
    return losses, opt


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--hidden", type=int, default=704)
    ap.add_argument("--blocks", type=int, default=2)
    a = ap.parse_args()
    torch.manual_seed(0)
    model = Stack(a.width, a.hidden, a.blocks)
    losses, opt = train(model, a.steps, a.width)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}; optimizer state {opt.mean_bits():.1f} bits a value; "
          f"saved for the backward pass {sum(b.saved_bytes(512) for b in model.blocks)} bytes at 512 tokens")
    with torch.no_grad():
        x = torch.randn(4, a.width, device="cuda").bfloat16()
        together = model(x)
        for b in model.blocks:
            b.freeze()
        one_by_one = torch.cat([model(x[i:i + 1]) for i in range(4)])
    print("served one token at a time: the same" if torch.equal(together, one_by_one) else "served one token at a time: DIFFERENT")


if __name__ == "__main__":
    main()
