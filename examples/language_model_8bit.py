"""A small language model trained and served with everything that the framework has for it.

An embedding, feed-forward blocks that save their state in 8 bits (FeedForward8), and an output layer that shares the embedding's matrix and
never holds the logits (VocabLoss); gradients clipped to a global norm inside the quantized optimizer's step (STQAdamW(max_norm=...)).
Afterwards tokens are scored one at a time.  (Without attention it learns which token follows which.)

    python examples/language_model_8bit.py [--steps 40] [--width 128] [--vocab 1003] [--blocks 2]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_06836_b200.ffn8 import FeedForward8  # noqa: E402
from paper_2604_06836_b200.head import VocabLoss  # noqa: E402
from paper_2604_06836_b200.optim import STQAdamW  # noqa: E402


class Model(torch.nn.Module):
    def __init__(self, vocab, width, blocks):
        super().__init__()
        self.embedding = torch.nn.Embedding(vocab, width, device="cuda")
        torch.nn.init.normal_(self.embedding.weight, std=0.1)
        self.blocks = torch.nn.ModuleList(FeedForward8(width, 3 * width) for _ in range(blocks))
        self.head = VocabLoss(width, vocab, weight=self.embedding.weight)

    def hidden(self, tokens):
        x, h = self.embedding(tokens).bfloat16(), None
        for b in self.blocks:
            x, h = b(x, h)
        return x + h

    def forward(self, tokens):
        """Mean loss of each token's successor; the last token of a sequence has none."""
        follows = torch.cat([tokens[:, 1:], torch.full_like(tokens[:, :1], self.head.ignore_index)], dim=1)
        return self.head(self.hidden(tokens), follows)

    def freeze(self):
        for m in (*self.blocks, self.head):
            m.freeze()
        return self


def batch(vocab, rows, length, gen):
    """Sequences in which a token is followed by one of three."""
    t = torch.randint(0, vocab, (rows, 1), device="cuda", generator=gen)
    out = [t]
    for _ in range(length - 1):
        t = (t * 7 + 3 + torch.randint(0, 3, t.shape, device="cuda", generator=gen)) % vocab
        out.append(t)
    return torch.cat(out, dim=1)


def train(model, steps, vocab, rows=32, length=64, lr=3e-3, max_norm=1.0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    opt = STQAdamW(model.parameters(), lr=lr, weight_decay=0.0, policy="paper", interval=10, max_norm=max_norm)
    losses, norms = [], []
    for _ in range(steps):
        opt.zero_grad()
        loss = model(batch(vocab, rows, length, gen))
        loss.backward()
        opt.step()
        losses.append(loss.detach())
        norms.append(opt.last_norm)
    return torch.stack(losses).tolist(), torch.stack(norms).tolist(), opt


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--vocab", type=int, default=1003)
    ap.add_argument("--blocks", type=int, default=2)
    a = ap.parse_args()
    torch.manual_seed(0)
    model = Model(a.vocab, a.width, a.blocks)
    losses, norms, opt = train(model, a.steps, a.vocab)
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f}; norm of the gradients {norms[0]:.2f} -> {norms[-1]:.2f}, clipped to 1; "
          f"optimizer state {opt.mean_bits():.1f} bits a value")
    with torch.no_grad():
        tokens = batch(a.vocab, 1, 16, torch.Generator(device="cuda").manual_seed(1))[0]
        model.freeze()
        scores = [float(model.head.scores(model.hidden(tokens[i:i + 1]), tokens[i + 1:i + 2])) for i in range(15)]
    print("log probabilities of a sequence, token by token:", " ".join(f"{s:.2f}" for s in scores))


if __name__ == "__main__":
    main()
