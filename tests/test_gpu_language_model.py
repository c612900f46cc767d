"""The output layer, the gradient norm and the quantized optimizer together, as a training program uses them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2604_06836_b200 import clip   # noqa: E402
from paper_2604_06836_b200.head import VocabLoss   # noqa: E402
from paper_2604_06836_b200.optim import STQAdamW   # noqa: E402

BF = torch.bfloat16


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "language_model_8bit.py")
    spec = importlib.util.spec_from_file_location("language_model_8bit", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def near(got, want, rel):
    off = float((got.detach().double() - want.detach()).norm() / want.detach().norm())
    assert off <= rel, off


def test_the_example_runs_and_its_gradients_are_right():
    """The shared matrix gets the gradient of the output layer and that of the embedding.  The first is held against 64 bits at the same
    hidden states; the second is the hidden states' gradient carried back through the blocks, by the same blocks."""
    e = example()
    torch.manual_seed(1)
    vocab, width = 301, 64
    model = e.Model(vocab, width, 2)
    tokens = e.batch(vocab, 8, 24, torch.Generator(device="cuda").manual_seed(3))
    model(tokens).backward()
    got = model.embedding.weight.grad.clone()

    for p in model.parameters():
        p.grad = None
    hidden = model.hidden(tokens)
    x = hidden.detach().double().reshape(-1, width).requires_grad_(True)
    w = model.embedding.weight.detach().to(BF).double().requires_grad_(True)
    follows = torch.cat([tokens[:, 1:], torch.full_like(tokens[:, :1], -100)], dim=1)
    torch.nn.functional.cross_entropy(x @ w.T, follows.reshape(-1)).backward()
    hidden.backward(x.grad.to(BF).view(hidden.shape))
    # the hidden states' gradient is rounded to bf16 in both (2^-8 at most each); what the blocks make of it is in 8 bits and bf16
    near(got, w.grad + model.embedding.weight.grad.double(), 0.02)

    losses, norms, opt = e.train(model, 12, vocab, rows=8, length=24)
    assert len(losses) == 12 and all(torch.isfinite(torch.tensor(losses + norms))) and opt.t == 12
    with torch.no_grad():
        model.freeze()
        both = model.head.scores(model.hidden(tokens[0, :4]), tokens[0, 1:5])
        one = torch.cat([model.head.scores(model.hidden(tokens[0, i:i + 1]), tokens[0, i + 1:i + 2]) for i in range(4)])
        near(one, both.double(), 1e-5)


@pytest.mark.parametrize("bias", [False, True])
def test_a_step_against_the_library(bias):
    """Loss, gradients, clipping and the update with 32-bit states, against torch's own in 64 bits, from the same weights.  The gradients are
    sums in fp32 (1e-5 in the 2-norm is their tests' bound); AdamW's first steps divide a gradient by its own size, so where one is
    smaller than that error its update is as uncertain as a whole step: the weights are compared in the 2-norm of the change."""
    torch.manual_seed(5)
    vocab, width, tokens = 501, 96, 400
    head = VocabLoss(width, vocab, bias)
    start = [p.detach().clone() for p in head.parameters()]
    opt = STQAdamW(head.parameters(), lr=1e-3, weight_decay=0.1, policy="fixed", init_bits=32, max_norm=0.05)
    ours = [p.detach().double().requires_grad_(True) for p in head.parameters()]
    lib = torch.optim.AdamW(ours, lr=1e-3, weight_decay=0.1)
    for step in range(4):
        h = torch.randn(tokens, width, device="cuda").to(BF)
        target = torch.randint(0, vocab, (tokens,), device="cuda")
        target[::7] = -100
        opt.zero_grad(), lib.zero_grad()
        loss = head(h, target)
        loss.backward()
        opt.step()
        w = ours[0].to(BF).double()      # (the products take the weight rounded; its gradient passes straight through)
        z = h.double() @ (ours[0] + (w - ours[0]).detach()).T + (ours[1] if bias else 0.0)
        want = torch.nn.functional.cross_entropy(z, target)
        want.backward()
        norm = torch.nn.utils.clip_grad_norm_(ours, 0.05)
        lib.step()
        assert abs(float(loss.detach()) - float(want.detach())) <= 1e-4 * float(want.detach())
        assert abs(float(opt.last_norm) - float(norm)) <= 1e-3 * float(norm)
        for p, q, s in zip(head.parameters(), ours, start):
            assert float((p.detach().double() - q.detach()).norm()) <= 0.02 * float((q.detach() - s.double()).norm())


def test_a_captured_step_trains_as_eager_ones_do():
    """Loss, gradients and the norm replayed from a graph, on new tokens in the same buffers, then the optimizer's step."""
    def make():
        torch.manual_seed(2)
        return VocabLoss(64, 300, True)

    data = [(torch.randn(200, 64, device="cuda").to(BF), torch.randint(-1, 300, (200,), device="cuda")) for _ in range(3)]
    eager = make()
    opt = STQAdamW(eager.parameters(), lr=1e-2, policy="fixed", init_bits=8, max_norm=0.1)
    eager.ignore_index = -1
    for h, t in data:
        opt.zero_grad()
        eager(h, t).backward()
        opt.step()

    m = make()
    m.ignore_index = -1
    opt2 = STQAdamW(m.parameters(), lr=1e-2, policy="fixed", init_bits=8, max_norm=0.1)
    h, t = data[0][0].clone(), data[0][1].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        warm = torch.autograd.grad(m(h, t), list(m.parameters()))
        clip.grad_norm(opt2.handle, warm, max_norm=0.1)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads = torch.autograd.grad(m(h, t), list(m.parameters()))
        norm = clip.grad_norm(opt2.handle, grads, max_norm=0.1)
    for p, g in zip(m.parameters(), grads):
        p.grad = g
    for a, b in data:
        h.copy_(a), t.copy_(b)
        graph.replay()
        opt2.step()
        assert torch.equal(opt2.last_norm, norm.norm)
    assert all(torch.equal(p, q) for p, q in zip(m.parameters(), eager.parameters()))
