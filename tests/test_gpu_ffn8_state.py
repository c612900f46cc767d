"""What the feed-forward block keeps, saves and refuses: weights in 8 bits, checkpoints, gradients nobody asked for."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2604_06836_b200 import ffn8, q8   # noqa: E402
from paper_2604_06836_b200.ffn8 import FeedForward8   # noqa: E402
from paper_2604_06836_b200.optim import STQAdamW   # noqa: E402

BF = torch.bfloat16


def block(width=72, hidden=136, kind="silu_gated", bias=False, seed=0):
    torch.manual_seed(seed)
    return FeedForward8(width, hidden, kind, bias)


def tokens(t=20, width=72, seed=1):
    return torch.randn(t, width, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(BF)


def served(m, x):
    with torch.no_grad():
        return m(x)[0]


# ---- streams ---------------------------------------------------------------------------------------------------------
def test_backward_passes_on_two_streams():
    """Both passes use the block's workspace; neither may see the other's partial sums."""
    m = block(392, 1000, bias=True)
    xs = [tokens(t, 392, t).requires_grad_(True) for t in (1500, 1700)]
    dys = [tokens(t, 392, 7 * t) for t in (1500, 1700)]

    def gradients(y, x, dy):
        return torch.autograd.grad(y, [x, *m.parameters()], dy)
    want = [gradients(m(x)[0], x, dy) for x, dy in zip(xs, dys)]
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(5):
        ys = []
        for s, x in zip(streams, xs):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                ys.append(m(x)[0])
        torch.cuda.synchronize()
        got = []
        for s, y, x, dy in zip(streams, ys, xs, dys):
            with torch.cuda.stream(s):
                got.append(gradients(y, x, dy))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            for u, v in zip(a, b):
                assert torch.equal(u, v)
    m.handle_for(xs[0].device).device_status()


# ---- derivatives -----------------------------------------------------------------------------------------------------
def test_a_second_derivative_is_refused():
    """The kernels leave no graph behind them: differentiating their gradients again must not pass for a constant."""
    m, x = block(), tokens().requires_grad_(True)
    y, h = m(x)
    for dy in (torch.ones_like(y), torch.ones_like(y).requires_grad_(True)):
        (g,) = torch.autograd.grad(y, x, dy, create_graph=True, retain_graph=True)
        with pytest.raises(RuntimeError, match="second"):
            (g.float().square().sum() + x.float().square().sum()).backward(retain_graph=True)
    (plain,) = torch.autograd.grad(y, x, torch.ones_like(y))
    assert torch.equal(plain, g)                          # the first derivative is as it was


def test_no_gradient_is_formed_that_nobody_asked_for(monkeypatch):
    count = {}
    for name in ("linear_dw", "linear_dx", "bias_grad", "norm_backward", "act_backward"):
        def call(*a, _real=getattr(q8, name), _name=name, **kw):
            count[_name] = count.get(_name, 0) + 1
            return _real(*a, **kw)
        monkeypatch.setattr(q8, name, call)
    m, x = block(bias=True), tokens().requires_grad_(True)
    m(x)[0].float().square().sum().backward()
    full = x.grad
    assert count == {"linear_dw": 2, "linear_dx": 2, "bias_grad": 2, "norm_backward": 1, "act_backward": 1}
    dw = m.w_out.grad

    count.clear()                                         # frozen weights: the input's gradient only
    m.requires_grad_(False)
    x.grad = None
    m(x)[0].float().square().sum().backward()
    assert torch.equal(x.grad, full)
    assert count == {"linear_dx": 2, "norm_backward": 1, "act_backward": 1}

    count.clear()                                         # the last product's weight only
    m.w_out.requires_grad_(True)
    m.w_out.grad = None
    m(x.detach())[0].float().square().sum().backward()
    assert torch.equal(m.w_out.grad, dw) and count == {"linear_dw": 1}

    count.clear()                                         # the first product's too: up to z, and no further
    m.w_in.requires_grad_(True)
    m(x.detach())[0].float().square().sum().backward()
    assert m.w_in.grad is not None and count == {"linear_dw": 2, "linear_dx": 1, "act_backward": 1}


# ---- what a pass saves -----------------------------------------------------------------------------------------------
def test_nothing_is_saved_where_no_gradient_is_taken(monkeypatch):
    asked = []

    def act(*a, _real=q8.act, **kw):
        asked.append(bool(kw.get("checkpoint")))
        return _real(*a, **kw)
    monkeypatch.setattr(q8, "act", act)
    m, x = block(), tokens()
    y = m(x)[0]
    assert asked == [True] and y.requires_grad
    with torch.no_grad():
        assert torch.equal(m(x)[0], y) and torch.equal(m.freeze()(x)[0], y)
    with torch.inference_mode():
        assert torch.equal(m(x)[0], y)
    m.requires_grad_(False)
    assert not m(x)[0].requires_grad
    assert asked == [True] + [False] * 4


# ---- frozen weights ----------------------------------------------------------------------------------------------------
def test_a_frozen_block_serves_the_weights_it_has():
    x = tokens()
    other = block(seed=5)
    want = served(other, x)

    m = block().freeze()
    m.load_state_dict(other.state_dict())
    assert torch.equal(served(m, x), want)
    m = block().freeze()
    m.load_state_dict({k: v.clone() for k, v in other.state_dict().items()}, assign=True)
    assert torch.equal(served(m, x), want)
    m = block().freeze()
    m.w_in, m.w_out = other.w_in, other.w_out
    assert torch.equal(served(m, x), want)
    m = block().freeze()
    with torch.no_grad():
        for p, q in zip(m.parameters(), other.parameters()):
            p.copy_(q)
    assert torch.equal(served(m, x), want)
    kept = m.weights8
    assert kept is not None and torch.equal(served(m, x), want) and m.weights8 is kept      # (quantized once, then kept)
    m.cpu()
    m.cuda()
    assert torch.equal(served(m, x), want)


def test_frozen_weights_on_another_stream_and_in_a_graph():
    x = tokens()
    m, other = block(1600, 3000), block(1600, 3000, seed=5)
    x = tokens(4, 1600)
    want, want2 = served(m, x), served(other, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        m.freeze()                                        # here; used there at once
        with torch.cuda.stream(side):
            got = served(m, x)
        side.synchronize()
        assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = served(m, x)
    m.load_state_dict(other.state_dict())
    assert torch.equal(served(m, x), want2)
    fill = [torch.full((1 << 20,), 7, dtype=torch.int8, device="cuda") for _ in range(32)]
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(captured, want)                    # the graph serves what it was captured with
    m.load_state_dict(block(1600, 3000).state_dict())
    with torch.cuda.graph(torch.cuda.CUDAGraph()):        # weights that changed before a capture are quantized in it
        captured = served(m, x)
    assert torch.equal(served(m, x), want) and len(fill) == 32
    with torch.inference_mode():
        m.load_state_dict(other.state_dict())
        assert torch.equal(m(x)[0], want2)
    m.requires_grad_(False)                               # codes that were made there can be saved here
    xg = x.clone().requires_grad_(True)
    m(xg)[0].float().sum().backward()
    assert float(xg.grad.abs().max()) > 0


def test_a_frozen_block_is_trained_on_its_weights():
    """A pass that differentiates the weights quantizes them as they are, frozen or not; what it serves afterwards is new."""
    x = tokens()
    a, b = block(), block().freeze()
    for m in (a, b):
        opt = STQAdamW(m.parameters(), lr=1e-2, weight_decay=0.0, policy="fixed", init_bits=8)
        for _ in range(3):
            opt.zero_grad()
            m(x)[0].float().square().sum().backward()
            opt.step()
    for p, q in zip(a.parameters(), b.parameters()):
        assert torch.equal(p, q)
    assert torch.equal(served(a, x), served(b, x))


def test_a_step_of_the_quantized_optimizer_reaches_a_frozen_block():
    x = tokens()
    m = block()
    opt = STQAdamW(m.parameters(), lr=1e-2, weight_decay=0.0, policy="fixed", init_bits=8)
    m(x)[0].float().square().sum().backward()
    before = served(m.freeze(), x)
    opt.step()
    after = served(m, x)
    assert not torch.equal(after, before) and torch.equal(after, served(m.thaw(), x))
    v = m.w_in._version
    opt.step()
    assert m.w_in._version > v                            # torch sees the change too


# ---- layouts -----------------------------------------------------------------------------------------------------------
def test_activations_in_any_layout():
    m, x, r = block(), tokens(24), tokens(24, seed=2)
    y, h = m(x, r)
    wide = torch.zeros(24, 80, device="cuda", dtype=BF)
    wide[:, :72] = x
    for v in (x.t().contiguous().t(), wide[:, :72], x.view(2, 3, 4, 72).permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3)):
        yv, hv = m(v, r.view(v.shape))
        assert yv.shape == v.shape and torch.equal(yv.reshape(24, 72), y) and torch.equal(hv.reshape(24, 72), h)
    one = x[:1].clone().requires_grad_(True)              # one residual row for all tokens
    ye, he = m(x, one.expand(24, 72))
    assert torch.equal(ye, m(x, one.detach().repeat(24, 1))[0])
    he.float().sum().backward()
    assert torch.equal(one.grad, torch.full_like(one, 24.0))
    assert torch.equal(m(x.t().contiguous().t())[1], x)


# ---- failures ----------------------------------------------------------------------------------------------------------
def test_a_wait_that_ran_out_is_reported_by_the_next_call():
    from paper_2604_06836_b200 import stq
    m, x = block(), tokens()
    m(x)
    hd = m.handle_for(x.device)
    hd.selftest_wait_timeout()
    torch.cuda.synchronize()
    with pytest.raises(stq.StqError) as e:
        m(x)
    assert e.value.code == -11
    with pytest.raises(stq.StqError) as e:
        q8.bias_grad(hd, x)
    assert e.value.code == -11
    assert served(block(), x).shape == x.shape            # a fresh handle works
