"""The output layer with its loss as a module: gradients, reductions, serving, streams, and a small model trained with it."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2604_06836_b200.head import VocabLoss   # noqa: E402

BF, F32 = torch.bfloat16, torch.float32
UB = 2.0 ** -8


def make(t=300, d=128, v=700, bias=True, dtype=F32, seed=1):
    torch.manual_seed(seed)
    weight = torch.nn.Parameter((torch.randn(v, d, device="cuda") / d ** 0.5).to(dtype))
    m = VocabLoss(d, v, bias, weight=weight)
    if bias:
        torch.nn.init.normal_(m.bias, std=0.1)
    h = torch.randn(t, d, device="cuda").to(BF).requires_grad_(True)
    target = torch.randint(0, v, (t,), device="cuda")
    target[torch.rand(t, device="cuda") < 0.2] = -100
    return m, h, target


def definition(m, h, target, reduction):
    """In 64 bits, from the weight as the products take it."""
    x = h.detach().double().requires_grad_(True)
    w = m.weight.detach().to(BF).double().requires_grad_(True)
    b = None if m.bias is None else m.bias.detach().double().requires_grad_(True)
    z = x.reshape(-1, x.shape[-1]) @ w.T
    loss = torch.nn.functional.cross_entropy(z if b is None else z + b, target.reshape(-1), ignore_index=-100, reduction=reduction)
    return loss, x, w, b


def near(got, want, rel):
    off = float((got.detach().double() - want.detach()).norm() / want.detach().norm())
    assert off <= rel, off


@pytest.mark.parametrize("dtype,bias", [(F32, True), (BF, False)])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_gradients(reduction, dtype, bias):
    """dx and a bf16 dw: two roundings to bf16 (UB each at most); an fp32 dw and dbias: sums in fp32."""
    m, h, target = make(bias=bias, dtype=dtype)
    loss = m(h, target, reduction)
    want, x, w, b = definition(m, h, target, reduction)
    near(loss, want, 1e-5)
    g = torch.randn_like(loss)
    loss.backward(g)
    want.backward(g.double())
    assert m.weight.grad.dtype == dtype
    near(h.grad, x.grad, 2 * UB)
    near(m.weight.grad, w.grad, 1e-5 if dtype == F32 else 2 * UB)
    if bias:
        near(m.bias.grad, b.grad, 1e-5)


def test_shapes_layouts_and_frozen_parts():
    m, h, target = make(t=24)
    flat = m(h, target, "none")
    for shape in ((4, 6), (2, 3, 4)):
        x = h.detach().view(*shape, -1)
        assert torch.equal(m(x, target.view(shape), "none"), flat.view(shape))
        t = x.transpose(0, 1)
        assert torch.equal(m(t, target.view(shape).transpose(0, 1), "none"), flat.view(shape).transpose(0, 1))
    wide = torch.zeros(24, 256, device="cuda", dtype=BF)
    wide[:, 1::2] = h.detach()
    assert torch.equal(m(wide[:, 1::2], target, "none"), flat)
    m.weight.requires_grad_(False)
    m(h, target).backward()
    assert m.weight.grad is None and h.grad is not None and m.bias.grad is not None
    m.bias.requires_grad_(False)
    assert not m(h.detach(), target).requires_grad


def test_no_token_counts():
    m, h, target = make()
    loss = m(h, torch.full_like(target, -100))
    loss.backward()
    assert float(loss.detach()) == 0.0 and all((p.grad == 0).all() for p in (h, m.weight, m.bias))


def test_scores_and_freezing():
    m, h, target = make()
    want = -m(h, target, "none").detach()
    assert torch.equal(m.scores(h, target), want)
    one = torch.cat([m.scores(h[i:i + 1], target[i:i + 1]) for i in range(20)])
    near(one, want[:20].double(), 1e-5)
    m.freeze()
    assert torch.equal(m.scores(h, target), want) and torch.equal(m.scores(h, target), want)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = m.scores(h, target)
    s.synchronize()
    assert torch.equal(other, want)
    with torch.no_grad():
        m.weight.mul_(2.0)      # a change that torch counts
    changed = m.scores(h, target)
    assert not torch.equal(changed, want) and torch.equal(changed, -m.thaw()(h, target, "none").detach())
    with torch.inference_mode():
        assert torch.equal(m.freeze().scores(h, target), changed)
    graph = torch.cuda.CUDAGraph()
    m.scores(h, target)
    with torch.cuda.graph(graph):
        out = m.scores(h, target)
    m.thaw()
    graph.replay()
    assert torch.equal(out, changed)


def test_streams_take_their_turns():
    m, h, target = make(t=2000, d=256, v=9000)
    want = torch.autograd.grad(m(h, target), [h, m.weight])
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 3]):
            got.append(torch.autograd.grad(m(h, target), [h, m.weight]))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_a_captured_training_pass():
    m, h, target = make()
    x, to = h.detach().clone().requires_grad_(True), target.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.autograd.grad(m(x, to), [x, m.weight, m.bias])
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = m(x, to)
        grads = torch.autograd.grad(loss, [x, m.weight, m.bias])
        loss = loss.detach()
    for seed in (3, 4):
        torch.manual_seed(seed)
        with torch.no_grad():
            x.copy_(torch.randn_like(x)), to.copy_(torch.randint(-1, 700, (300,), device="cuda"))
            to[to < 0] = -100
        graph.replay()
        got = [v.clone() for v in (loss, *grads)]
        eager = m(x, to)
        for a, b in zip(got, (eager, *torch.autograd.grad(eager, [x, m.weight, m.bias]))):
            assert torch.equal(a, b)


def test_second_derivatives_are_refused():
    m, h, target = make()
    (g,) = torch.autograd.grad(m(h, target), [h], create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        g.float().sum().backward()


def test_a_copy_and_a_move():
    import copy
    m, h, target = make()
    want = m.freeze().scores(h, target)
    c = copy.deepcopy(m)
    assert torch.equal(c.scores(h, target), want)
    c.load_state_dict({k: v * 0.5 for k, v in m.state_dict().items()})
    assert not torch.equal(c.scores(h, target), want)
