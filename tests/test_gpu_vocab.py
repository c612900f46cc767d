"""Cross entropy over a vocabulary and its gradients (stq_vocab_*) against the definition in 64 bits, element by element.

Tolerances.  U = 2^-24 and UB = 2^-8 are half steps of fp32 and bf16.  A logit is a sum of d products formed 16 at a time in fp32, each
addition cut off (one step, 2 U) and the products exact: it is off by dz <= 2 U (d / 16 + 2) a with a = the sum of the products'
magnitudes.  lse is off by the largest dz of the row and by the roundings of exp, of a sum that is joined in a few hundred steps of
which at most 2 v / 128 + 64 follow one another, and of log.  A gradient of a logit g (p - [hit]) is off by g p e with
e = dz + error of lse + 8 U (|z - lse| + 2), and by UB of itself where it is rounded to bf16.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2604_06836_b200 import stq, vocab   # noqa: E402

BF, F32 = torch.bfloat16, torch.float32
U, UB = 2.0 ** -24, 2.0 ** -8
IGNORE = -100


@pytest.fixture(scope="module")
def handle():
    h = stq.Handle()
    yield h
    h.device_status()
    h.close()


def pitched(x, extra, shift=0, fill=7.0):
    """The same matrix with `extra` more elements to a row, beginning `shift` elements into the buffer."""
    r, c = x.shape
    buf = torch.full((r * (c + extra) + shift + 64,), fill, device=x.device, dtype=torch.float32).to(x.dtype)
    v = buf[shift:shift + r * (c + extra)].view(r, c + extra)[:, :c]
    v.copy_(x)
    return v


def inputs(t, d, v, seed, bias=False, masked=0.0, sharp=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)      # noqa: E731
    x = rand(t, d).to(BF)
    w = (rand(v, d) * (sharp / d ** 0.5)).to(BF)
    target = torch.randint(0, v, (t,), device="cuda", generator=g)
    target[torch.rand(t, device="cuda", generator=g) < masked] = IGNORE
    b = 0.5 * rand(v) if bias else None
    return x, w, target, b, rand(t) * 1e-3


class Definition:
    """Everything in 64 bits, with the bounds of the docstring."""

    def __init__(self, x, w, target, b, dloss, ignore=IGNORE):
        x, w = x.double(), w.double()
        t, d = x.shape
        v = w.shape[0]
        self.counts = target != ignore
        z = x @ w.T + (0.0 if b is None else b.double())
        a = x.abs() @ w.abs().T + (0.0 if b is None else b.double().abs())
        dz = 2 * U * (d / 16 + 2) * a + U * z.abs()
        lse = torch.logsumexp(z, 1)
        self.elog = dz.amax(1) + 8 * U * (lse.abs() + (z - lse[:, None]).abs().amax(1)) + U * (2 * v / 128 + 64)
        at = torch.where(self.counts, target, 0)[:, None]
        self.lse = torch.where(self.counts, lse, 0.0)
        self.loss = torch.where(self.counts, lse - z.gather(1, at)[:, 0], 0.0)
        self.eloss = self.elog + dz.gather(1, at)[:, 0] + 2 * U * (self.loss.abs() + lse.abs())
        p = torch.softmax(z, 1)
        g = torch.where(self.counts, dloss.double(), 0.0)[:, None]
        e = dz + self.elog[:, None] + 8 * U * ((z - lse[:, None]).abs() + 2)
        grad = p.scatter_add(1, at, -torch.ones_like(p[:, :1])) * g
        off = p * e * g.abs()
        self.x, self.w, self.grad, self.off = x, w, grad, off
        self.t, self.v = t, v

    def check(self, out, grads, dtype, what=""):
        def near(got, want, tol, name):
            got = got.double()
            assert got.shape == want.shape, (what, name)
            bad = ~((got - want).abs() <= tol)
            assert not bad.any(), (what, name, float(((got - want).abs() / tol).nan_to_num(nan=1e30).max()), bad.nonzero()[:4].tolist())
        near(out.lse, self.lse, torch.where(self.counts, self.elog, 0.0), "lse")
        near(out.loss, self.loss, torch.where(self.counts, self.eloss, 0.0), "loss")
        if grads is None:
            return
        mag, x, w = self.grad.abs(), self.x, self.w
        rounded = UB * mag + self.off
        if grads.dx is not None:
            want = self.grad @ w      # sums of v / 16 steps, joined over pieces, pairs and planes
            near(grads.dx, want, (UB * want.abs() + (rounded @ w.abs()) * (1 + UB) + 2 * U * (self.v / 16 + 64) * (mag @ w.abs())) + 1e-44, "dx")
            assert (grads.dx[~self.counts] == 0).all()
        if grads.dw is not None:
            want, size = self.grad.T @ x, mag.T @ x.abs()
            if dtype == F32:          # 24 products of 16 to a chunk of 128 terms, then one rounded addition a chunk
                tol = self.off.T @ x.abs() + 2 * U * (24 + self.t / 128 + 34) * size + U * want.abs()
            else:
                tol = UB * want.abs() + (rounded.T @ x.abs()) * (1 + UB) + 2 * U * (self.t / 16 + 34) * size
            near(grads.dw, want, tol + 1e-44, "dw")
        if grads.dbias is not None:
            near(grads.dbias, self.grad.sum(0), self.off.sum(0) + U * (self.t / 8 + 32) * mag.sum(0) + 1e-44, "dbias")


def run(handle, x, w, target, b, dloss, dtype, **kw):
    out = vocab.loss(handle, x, w, target, bias=b)
    return out, vocab.loss_backward(handle, dloss, x, w, target, out.lse, bias=b, dtype=dtype, **kw)


SIZES = [(1, 1, 1), (1, 64, 100), (1, 1600, 1283), (2, 8, 2), (3, 77, 131), (61, 769, 1283), (128, 256, 1000), (129, 72, 257),
         (130, 65, 511), (200, 64, 100), (257, 1025, 5121), (512, 768, 1000), (1003, 136, 3001), (300, 1600, 20001), (2500, 200, 900),
         (5000, 32, 77)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("t,d,v", SIZES)
def test_loss_and_gradients(handle, t, d, v, dtype):
    for bias, masked in ((False, 0.0), (True, 0.3)):
        x, w, target, b, dloss = inputs(t, d, v, t + d + v, bias, masked)
        out, grads = run(handle, x, w, target, b, dloss, dtype)
        Definition(x, w, target, b, dloss).check(out, grads, dtype, f"{t} {d} {v} {bias}")
