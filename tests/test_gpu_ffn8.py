"""The feed-forward block that saves its state in 8 bits: gradients, training with the quantized optimizer, serving."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2604_06836_b200 import q8   # noqa: E402
from paper_2604_06836_b200.ffn8 import FeedForward8   # noqa: E402

BF = torch.bfloat16


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "feed_forward_8bit.py")
    spec = importlib.util.spec_from_file_location("feed_forward_8bit", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


class Through(torch.autograd.Function):
    """Straight through a rounding: `to` forwards, the gradient of `x` backwards."""
    @staticmethod
    def forward(ctx, x, to):
        return to

    @staticmethod
    def backward(ctx, g):
        return g, None


@pytest.mark.parametrize("kind,bias", [("silu_gated", False), ("gelu", True)])
@pytest.mark.parametrize("with_residual", [True, False])
def test_gradients_against_64_bits(kind, bias, with_residual):
    """The block's formulas in 64 bits around the same 8-bit values, differentiated by autograd.  What is left is the
    rounding of z, of the gradients between the operators and of the operands to bf16: each 2^-8 of its terms at most, far
    less in the 2-norm, where 2 % covers the five of them in a row."""
    torch.manual_seed(3)
    t, d, f = 200, 136, 264
    m = FeedForward8(d, f, kind, bias)
    if bias:
        torch.nn.init.normal_(m.b_in, std=0.1), torch.nn.init.normal_(m.b_out, std=0.1)
    torch.nn.init.normal_(m.weight, mean=1.0, std=0.1)
    x = torch.randn(2, t // 2, d, device="cuda").to(BF).requires_grad_(True)
    r = torch.randn(2, t // 2, d, device="cuda").to(BF).requires_grad_(True) if with_residual else None
    gy, gh = torch.randn(t, d, device="cuda").to(BF), torch.randn(t, d, device="cuda").to(BF)
    y, h = m(x, r)
    ((y.reshape(t, d) * gy).sum() + (h.reshape(t, d) * gh).sum()).backward()

    hd = m.handle_for(x.device)
    p = {n: v.detach().double().requires_grad_(True) for n, v in m.named_parameters()}
    xd = x.detach().double().reshape(t, d).requires_grad_(True)
    rd = r.detach().double().reshape(t, d).requires_grad_(True) if with_residual else None
    n8 = q8.norm(hd, x.detach().reshape(t, d), m.weight.detach(), residual=None if r is None else r.detach().reshape(t, d))
    w_in, w_out = (w.values(torch.float64) for w in m.quantized())
    hh = xd + rd if with_residual else xd
    n = hh * (hh.square().mean(1, keepdim=True) + m.eps).rsqrt() * p["weight"]
    z = Through.apply(n, n8.rows.values(torch.float64)) @ Through.apply(p["w_in"], w_in).T
    z = z + p["b_in"] if bias else z
    a8 = q8.act(hd, z.detach().to(BF), kind, checkpoint=True)
    zq = Through.apply(z, a8.checkpoint.values().double())
    a = zq[:, :f] * torch.sigmoid(zq[:, :f]) * zq[:, f:] if kind == "silu_gated" else torch.nn.functional.gelu(zq, approximate="tanh")
    yy = Through.apply(a, a8.rows.values(torch.float64)) @ Through.apply(p["w_out"], w_out).T
    yy = yy + p["b_out"] if bias else yy
    ((yy * gy.double()).sum() + (hh * gh.double()).sum()).backward()

    def near(got, want, what):
        rel = float((got.detach().double() - want.detach()).norm() / want.detach().norm())
        assert rel <= 0.02, (what, rel)
    near(y.reshape(t, d), yy, "y")
    near(x.grad.reshape(t, d), xd.grad, "dx")
    if with_residual:
        assert torch.equal(x.grad, r.grad)
    for name, v in m.named_parameters():
        assert v.grad.dtype == torch.float32
        near(v.grad, p[name].grad, name)


def test_refusals():
    with pytest.raises(ValueError, match="kind"):
        FeedForward8(64, 64, "relu")
    with pytest.raises(ValueError, match="bfloat16"):
        FeedForward8(64, 64)(torch.zeros(2, 64, device="cuda"))


def test_saved_state_is_small():
    import copy
    m = FeedForward8(1600, 6400)
    x = torch.randn(3, 1600, device="cuda").to(BF)
    y = m(x)[0].detach()
    assert torch.equal(copy.deepcopy(m)(x)[0].detach(), y)      # (with a handle of its own)
    assert m.saved_bytes(1) < 0.53 * 2 * (1600 + 3 * 6400)


@pytest.mark.parametrize("kind", ["silu_gated", "gelu"])
def test_training_with_the_quantized_optimizer_and_serving(kind):
    ex = example()
    torch.manual_seed(1)
    model = ex.Stack(128, 352, 2, kind)
    losses, opt = ex.train(model, 50, 128, tokens=256)
    assert sum(losses[-5:]) < 0.6 * sum(losses[:5])
    with torch.no_grad():
        x = torch.randn(40, 128, device="cuda").to(BF)
        whole = model(x)
        for b in model.blocks:
            b.freeze()
        assert torch.equal(model(x), whole)
        # integer sums are exact, so a token does not depend on what it is batched with
        assert torch.equal(torch.cat([model(x[i:i + 1]) for i in range(40)]), whole)
        assert torch.equal(model(x[:20]), whole[:20])
    for b in model.blocks:
        b.handle_for(x.device).device_status()
