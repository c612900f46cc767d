"""Cross entropy over a vocabulary and its gradients (stq_vocab_*) against the definition in 64 bits, element by element.

Tolerances.  U = 2^-24 and UB = 2^-8 are half steps of fp32 and bf16.  A logit is a sum of d products formed 16 at a time in fp32, each
addition cut off (one step, 2 U) and the products exact: it is off by dz <= 2 U (d / 16 + 2) a with a = the sum of the products'
magnitudes.  lse is off by the largest dz of the row and by the roundings of exp, of a sum that is joined in a few hundred steps of
which at most 2 v / 128 + 64 follow one another, and of log.  A gradient of a logit g (p - [hit]) is off by g p e with
e = dz + error of lse + 8 U (|z - lse| + 2), and by UB of itself where it is rounded to bf16.  Below the normal numbers, 2^-126, all
of this is absolute: an exp that is smaller may come out as 0, which g carries on, and so may the product with g and each of the three
parts that it is passed on in: (|g| + 4) 2^-126.
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
        off = p * e * g.abs() + (g.abs() + 4) * 2.0 ** -126 * (g != 0)
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


@pytest.mark.parametrize("d", [1, 7, 8, 33, 250, 1000, 1024, 1032, 1601, 2050, 4096, 5000])
@pytest.mark.parametrize("t", [1, 3, 8, 9, 16, 17])
def test_few_tokens(handle, t, d):
    """A tile of which most rows are not there."""
    for v in (1, 15, 16, 17, 250, 9001):
        x, w, target, b, dloss = inputs(t, d, v, t + d + v, v % 2 == 1, 0.2 if t > 2 else 0.0)
        out = vocab.loss(handle, x, w, target, bias=b)
        Definition(x, w, target, b, dloss).check(out, None, BF, f"{t} {d} {v}")
        wp, xp = pitched(w, 8 + (-d) % 8, 0, float("nan")), pitched(x, 3, 1, float("nan"))      # (rows of w stay aligned)
        again = vocab.loss(handle, xp, wp, target, bias=b)
        assert torch.equal(out.lse, again.lse)


@pytest.mark.parametrize("d", [77, 929, 4096])
@pytest.mark.parametrize("t", [1, 3, 40, 129, 700])
def test_loss_of_confident_tokens(handle, t, d):
    """Where the target has nearly all of the sum, the loss is much smaller than lse and the target's logit, and what these are off by must
    not show.  loss = log(1 + sum of exp(z_j - z_target) over the others): off by those terms' shares times their errors, by 11 additions
    to a sum that holds a 1 (32 entries: 8 to each of four sums, these joined, and joined to what there was), and by the roundings of
    log, of the difference and of the result."""
    v, g = 32, torch.Generator(device="cuda").manual_seed(t + d)
    w = (torch.randn(v, d, device="cuda", generator=g) * (2 / d ** 0.5)).to(BF)
    target = torch.randint(0, v, (t,), device="cuda", generator=g)
    sure = 1 + 3 * torch.rand(t, 1, device="cuda", generator=g)
    x = (0.3 * torch.randn(t, d, device="cuda", generator=g) + sure * w[target].float()).to(BF)
    if t > 3:
        target[::5] = IGNORE
    out = vocab.loss(handle, x, w, target)
    x, w, counts = x.double(), w.double(), target != IGNORE
    at = torch.where(counts, target, 0)[:, None]
    z, a = x @ w.T, x.abs() @ w.abs().T
    dz = 2 * U * (d / 16 + 2) * a + U * z.abs()
    apart = z - z.gather(1, at)
    others = torch.softmax(z, 1).scatter(1, at, 0.0)
    loss = torch.logsumexp(apart, 1)
    off = (others * (dz + dz.gather(1, at) + 8 * U * (apart.abs() + apart.amax(1, keepdim=True) + 2))).sum(1) + 11 * U + 4 * U * loss
    assert (out.loss[~counts] == 0).all() and (out.loss >= 0).all()
    bad = counts & ~((out.loss.double() - loss).abs() <= off)
    assert not bad.any(), ((out.loss.double() - loss)[bad], loss[bad])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("t,d,v", SIZES)
def test_loss_and_gradients(handle, t, d, v, dtype):
    for bias, masked in ((False, 0.0), (True, 0.3)):
        x, w, target, b, dloss = inputs(t, d, v, t + d + v, bias, masked)
        out, grads = run(handle, x, w, target, b, dloss, dtype)
        Definition(x, w, target, b, dloss).check(out, grads, dtype, f"{t} {d} {v} {bias}")


def test_many_pieces_of_the_vocabulary(handle):
    """The gradients of the logits of 9000 tokens exist for some 28000 entries at a time (9000 in three parts): two pieces, and four."""
    x, w, target, b, dloss = inputs(9000, 72, 30001, 5, True, 0.1)
    d = Definition(x, w, target, b, dloss)
    for dtype in (BF, F32):
        out, grads = run(handle, x, w, target, b, dloss, dtype)
        d.check(out, grads, dtype, "pieces")


def test_more_tokens_than_a_loss_takes_at_once(handle):
    x, w, target, b, dloss = inputs(70001, 16, 300, 6, True, 0.5)
    d = Definition(x, w, target, b, dloss)
    out, grads = run(handle, x, w, target, b, dloss, F32)
    d.check(out, grads, F32, "tokens")


@pytest.mark.parametrize("extra,shift", [(8, 0), (8, 8), (3, 0), (1, 1), (0, 3)])
@pytest.mark.parametrize("t", [5, 300])
def test_pitches_and_alignment(handle, t, extra, shift):
    x, w, target, b, dloss = inputs(t, 200, 333, 8, True, 0.2)
    want_out, want = run(handle, x, w, target, b, dloss, BF)
    for fill in (7.0, float("nan")):      # what lies between the rows does not matter
        xp, wp = pitched(x, extra, shift, fill), pitched(w, extra, shift, fill)
        out, grads = run(handle, xp, wp, target, b, dloss, BF)
        assert torch.equal(out.lse, want_out.lse) and torch.equal(grads.dx, want.dx) and torch.equal(grads.dw, want.dw)
        Definition(x, w, target, b, dloss).check(out, grads, BF, "pitch")


def test_which_gradients_are_asked_for(handle):
    x, w, target, b, dloss = inputs(300, 128, 700, 9, True, 0.2)
    out, want = run(handle, x, w, target, b, dloss, F32)
    for dx in (True, False):
        for dw in (True, False):
            for db in (True, False):
                g = vocab.loss_backward(handle, dloss, x, w, target, out.lse, bias=b, dtype=F32, want_dx=dx, want_dw=dw, want_dbias=db)
                for got, full, asked in zip(g, want, (dx, dw, db)):
                    assert (got is not None) == asked and (got is None or torch.equal(got, full))
    g = vocab.loss_backward(handle, dloss, x, w, target, out.lse, want_dbias=True)      # (of a bias of zeros)
    assert g.dbias.shape == (700,)


@pytest.mark.parametrize("t", [1, 100, 129, 700])
def test_no_token_counts(handle, t):
    x, w, target, b, dloss = inputs(t, 128, 300, 3, True)
    target.fill_(IGNORE)
    for dtype in (BF, F32):
        out, grads = run(handle, x, w, target, b, dloss, dtype)
        assert all((v == 0).all() for v in (*out, *grads))


def test_no_tokens(handle):
    x, w, target, b, dloss = inputs(0, 128, 300, 3, True)
    out, grads = run(handle, x, w, target, b, dloss, F32)
    assert out.loss.shape == (0,) and grads.dx.shape == (0, 128) and (grads.dw == 0).all() and (grads.dbias == 0).all()


@pytest.mark.parametrize("t", [100, 500])
def test_ignored_tokens_may_hold_anything(handle, t):
    """NaN, infinities and huge values of tokens without a loss reach nothing, nor does their dloss."""
    x, w, target, b, dloss = inputs(t, 128, 700, 4, True, 0.4)
    want_out, want = run(handle, x, w, target, b, dloss, F32)
    off = target == IGNORE
    for value in (float("nan"), float("inf"), 3e38):
        x2, d2 = x.clone(), dloss.clone()
        x2[off] = value
        d2[off] = value
        out, grads = run(handle, x2, w, target, b, d2, F32)
        assert all(torch.equal(a, c) for a, c in zip((*out, *grads), (*want_out, *want)))


def test_another_ignore_index(handle):
    x, w, target, b, dloss = inputs(300, 128, 700, 4, False, 0.4)
    want = vocab.loss(handle, x, w, target)
    other = torch.where(target == IGNORE, 5, torch.where(target == 5, 6, target))
    out = vocab.loss(handle, x, w, other, ignore_index=5)
    keep = target != 5
    assert torch.equal(out.lse[keep], want.lse[keep])


@pytest.mark.parametrize("t", [100, 500])
def test_targets_outside_the_vocabulary_give_nan(handle, t):
    x, w, target, b, dloss = inputs(t, 128, 700, 4, False, 0.2)
    want_out, want = run(handle, x, w, target, b, dloss, BF)
    for bad in (700, -1, -99, 2 ** 40, -2 ** 63):
        wrong = target.clone()
        wrong[17] = bad
        out, grads = run(handle, x, w, wrong, b, dloss, BF)
        assert out.loss[17].isnan() and out.lse[17].isnan() and grads.dx[17].isnan().all() and grads.dw.isnan().any()
        others = torch.arange(t, device="cuda") != 17
        assert torch.equal(out.loss[others], want_out.loss[others]) and torch.equal(grads.dx[others], want.dx[others])


@pytest.mark.parametrize("t", [12, 60, 400])
def test_entries_out_of_the_vocabulary(handle, t):
    """A bias of -inf, or of the lowest number: probability 0, no gradient, also where they fill whole tiles."""
    x, w, target, b, dloss = inputs(t, 64, 1500, 4, True)
    target = target % 300
    live = torch.arange(1500, device="cuda") < 300
    d = Definition(x, w[live], target, b[live], dloss)
    for low in (-float("inf"), -3.4e38):
        cut = torch.where(live, b, low)
        out, grads = run(handle, x, w, target, cut, dloss, F32)
        d.check(out, vocab.LossGrads(grads.dx, grads.dw[live], grads.dbias[live]), F32, str(low))
        assert (grads.dw[~live] == 0).all() and (grads.dbias[~live] == 0).all()
    # all of the vocabulary: there is nothing to normalise
    out = vocab.loss(handle, x, w, target, bias=torch.full_like(b, -float("inf")))
    assert (out.lse == -float("inf")).all() and out.loss.isnan().all()
    # a target that is out: its loss is infinite, the others are as they were
    wrong = target.clone()
    wrong[3] = 1400
    o = vocab.loss(handle, x, w, wrong, bias=torch.where(live, b, -float("inf")))
    assert o.loss[3] == float("inf") and torch.equal(o.lse[4:], vocab.loss(handle, x, w, target, bias=torch.where(live, b, -float("inf"))).lse[4:])


@pytest.mark.parametrize("t", [12, 60, 400])
def test_infinities_and_nan_stay_in_their_row(handle, t):
    x, w, target, b, dloss = inputs(t, 64, 900, 4)
    want_out, want = run(handle, x, w, target, b, dloss, BF)
    x = x.clone()
    x[5, 3], x[9, 0] = float("nan"), float("inf")
    out, grads = run(handle, x, w, target, b, dloss, BF)
    rows = torch.ones(t, dtype=torch.bool, device="cuda")
    rows[5] = rows[9] = False
    assert out.loss[5].isnan() and out.loss[9].isnan() and grads.dx[5].isnan().all()
    assert torch.equal(out.loss[rows], want_out.loss[rows]) and torch.equal(grads.dx[rows], want.dx[rows])


def test_logits_far_apart(handle):
    """Logits in the thousands: one entry has all of the probability."""
    x, w, target, b, dloss = inputs(300, 64, 900, 4, sharp=500.0)
    out, grads = run(handle, x, w, target, b, dloss, F32)
    Definition(x, w, target, b, dloss).check(out, grads, F32, "sharp")


def test_the_same_from_run_to_run(handle):
    x, w, target, b, dloss = inputs(700, 300, 3000, 4, True, 0.3)
    first = run(handle, x, w, target, b, dloss, F32)
    for _ in range(3):
        again = run(handle, x, w, target, b, dloss, F32)
        assert all(torch.equal(a, c) for p, q in zip(first, again) for a, c in zip(p, q))


def test_gradients_against_differences(handle):
    """The loss along +-2^-7 in w and in x, on numbers that bf16 holds exactly: (L+ - L-) / 2h is the derivative up to h^2 q^3, q the
    largest change of a logit per unit, and to the error of the two losses over 2h."""
    g = torch.Generator(device="cuda").manual_seed(2)
    t, d, v, h = 200, 32, 150, 2.0 ** -7
    pick = lambda n, m, a: torch.randint(-a, a + 1, (n, m), device="cuda", generator=g)      # noqa: E731
    x, w = (pick(t, d, 31) * 2.0 ** -6).to(BF), (pick(v, d, 31) * 2.0 ** -6).to(BF)
    ux, uw = pick(t, d, 1).float(), pick(v, d, 1).float()
    target = torch.randint(0, v, (t,), device="cuda", generator=g)
    dloss = torch.randn(t, device="cuda", generator=g)
    out, grads = run(handle, x, w, target, None, dloss, F32)
    total = lambda a, c: float((vocab.loss(handle, a, c, target).loss.double() * dloss.double()).sum())      # noqa: E731
    weight = float(dloss.abs().sum())
    for kind in ("w", "x"):
        at = lambda s: total(x, (w.float() + s * h * uw).to(BF)) if kind == "w" else total((x.float() + s * h * ux).to(BF), w)      # noqa: E731
        slope = (at(1) - at(-1)) / (2 * h)
        got = float((grads.dw.double() * uw).sum()) if kind == "w" else float((grads.dx.double() * ux).sum())
        change = (x.float() @ uw.T if kind == "w" else ux @ w.float().T).abs().max()
        tol = weight * float(h * h * change ** 3 + 64 * U / h) + (0 if kind == "w" else 2 * UB * float((grads.dx.double().abs() * ux.abs()).sum()))
        assert abs(got - slope) <= tol and tol < 0.2 * abs(slope) + 0.2 * weight, (kind, got, slope, tol)


def test_on_another_stream_and_in_a_graph(handle):
    x, w, target, b, dloss = inputs(500, 128, 2000, 4, True, 0.3)
    want = run(handle, x, w, target, b, dloss, BF)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    x2 = torch.zeros_like(x)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(2000000)
        x2.copy_(x)
    out = vocab.loss(handle, x2, w, target, bias=b, stream=s)
    grads = vocab.loss_backward(handle, dloss, x2, w, target, out.lse, bias=b, stream=s)
    s.synchronize()
    assert all(torch.equal(a, c) for p, q in zip(want, (out, grads)) for a, c in zip(p, q))

    hd = stq.Handle()      # (its workspace grows inside the capture)
    to = target.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, grads = run(hd, x2, w, to, b, dloss, BF)
    big = inputs(3000, 256, 5000, 5)
    run(hd, *big, F32)      # a larger call replaces the workspace; the graph keeps its own
    for masked in (0.0, 0.9):      # how many tokens count is read on the device
        new = inputs(500, 128, 2000, 11, True, masked)
        x2.copy_(new[0]), to.copy_(new[2])
        graph.replay()
        Definition(x2, w, to, b, dloss).check(out, grads, BF, f"graph {masked}")
    hd.device_status()
    del graph


def test_refusals(handle):
    x, w, target, b, dloss = inputs(10, 64, 100, 1, True)
    lse = dloss.clone()
    for call, what in ((lambda: vocab.loss(handle, x.float(), w, target), "bfloat16"),
                       (lambda: vocab.loss(handle, x, w.half(), target), "bfloat16"),
                       (lambda: vocab.loss(handle, x[:, :63], w, target), "63 columns"),
                       (lambda: vocab.loss(handle, x.T, w, target), "unit stride|columns"),
                       (lambda: vocab.loss(handle, x, w, target.int()), "int64"),
                       (lambda: vocab.loss(handle, x, w, target[:9]), "int64"),
                       (lambda: vocab.loss(handle, x, w, target, bias=b.to(BF)), "float32"),
                       (lambda: vocab.loss(handle, x, w.cpu(), target), "device"),
                       (lambda: vocab.loss_backward(handle, dloss[:9], x, w, target, lse), "dloss"),
                       (lambda: vocab.loss_backward(handle, dloss, x, w, target, lse.double()), "lse"),
                       (lambda: vocab.loss_backward(handle, dloss, x, w, target, lse, dtype=torch.float16), "dtype")):
        with pytest.raises(ValueError, match=what):
            call()
    with pytest.raises(stq.StqError) as e:
        vocab.loss(handle, x, w[:0], target)
    assert e.value.code == -6
    L, p = vocab._lib(), lambda t: t.data_ptr()      # noqa: E731
    out = torch.empty(10, device="cuda")
    assert L.stq_vocab_loss(handle._h, p(x), 64, p(w), 64, None, p(target), -100, 10, 100, 64, p(out), p(out), None) == -5
    assert L.stq_vocab_loss(handle._h, p(x), 63, p(w), 64, None, p(target), -100, 10, 100, 64, p(out), p(lse), None) == -9
    assert L.stq_vocab_loss(handle._h, p(x), 64, p(w), 64, None, None, -100, 10, 100, 64, p(out), p(lse), None) == -1
    assert L.stq_vocab_loss(handle._h, p(x), 64, p(w), 64, None, p(target), -100, 262145, 100, 64, p(out), p(lse), None) == -12
    assert L.stq_vocab_loss_backward(handle._h, p(dloss), p(x), 64, p(w), 64, None, p(target), -100, p(lse), 10, 100, 64, p(x), 64, None, 0, 0,
                                     None, None) == -5


def test_a_wait_that_ran_out_is_reported():
    """A handle with a launch behind it that gave up refuses both operators without synchronising."""
    from paper_2604_06836_b200 import clip
    hd = stq.Handle()
    x, w, target, b, dloss = inputs(10, 64, 100, 1)
    out = vocab.loss(hd, x, w, target)
    hd.selftest_wait_timeout()
    torch.cuda.synchronize()
    for call in (lambda: vocab.loss(hd, x, w, target), lambda: vocab.loss_backward(hd, dloss, x, w, target, out.lse),
                 lambda: clip.grad_norm(hd, [dloss])):
        with pytest.raises(stq.StqError) as e:
            call()
        assert e.value.code == -11
    hd.close()


def test_a_large_vocabulary_bounds_the_tokens_at_once(handle):
    """The parts of a loss fit 256 MB: of 600 000 entries 3400 tokens or so at a time, here in three blocks."""
    x, w, target, b, dloss = inputs(9001, 16, 600001, 3, True, 0.3, sharp=1.0)
    out = vocab.loss(handle, x, w, target, bias=b)
    for rows in (slice(0, 200), slice(3400, 3700), slice(8900, 9001)):
        Definition(x[rows], w, target[rows], b, dloss[rows]).check(vocab.LossOut(out.loss[rows], out.lse[rows]), None, BF, str(rows))
    whole = torch.cat([vocab.loss(handle, x[i:i + 2000], w, target[i:i + 2000], bias=b).lse for i in range(0, 9001, 2000)])
    assert float((whole - out.lse).abs().max()) <= 1e-5


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e30])
def test_dloss_of_any_size(handle, scale):
    """The logits' gradients are formed relative to the largest dloss, so its size does not matter to them."""
    x, w, target, b, dloss = inputs(200, 64, 300, 2, True, 0.2)
    out, want = run(handle, x, w, target, b, dloss, F32)
    big = vocab.loss_backward(handle, dloss * 1e3 * scale, x, w, target, out.lse, bias=b, dtype=F32)
    for a, c in ((big.dw, want.dw), (big.dbias, want.dbias)):
        assert float((a.double() / (1e3 * scale) - c.double()).abs().max()) <= 1e-6 * float(c.abs().max()) + 1e-45 / (1e3 * scale)


def test_dloss_of_zero_and_of_infinity(handle):
    x, w, target, b, dloss = inputs(200, 64, 300, 2, True)
    out = vocab.loss(handle, x, w, target, bias=b)
    zero = vocab.loss_backward(handle, torch.zeros_like(dloss), x, w, target, out.lse, bias=b, dtype=F32)
    assert all((g == 0).all() for g in zero)
    one = torch.zeros_like(dloss)
    one[7] = float("inf")
    g = vocab.loss_backward(handle, one, x, w, target, out.lse, bias=b, dtype=F32)
    rows = torch.arange(200, device="cuda") != 7
    assert (g.dx[rows] == 0).all() and not g.dx[7].isfinite().any()


def test_tokens_that_repeat(handle):
    """The same row many times, and one target for all: what adds up in dw adds up in order."""
    x, w, target, b, dloss = inputs(1, 72, 500, 2)
    x, target, dloss = x.repeat(1500, 1), target.repeat(1500), torch.full((1500,), 1 / 1500, device="cuda")
    out, grads = run(handle, x, w, target, b, dloss, F32)
    assert (out.loss == out.loss[0]).all() and (grads.dx == grads.dx[0]).all()
    Definition(x, w, target, b, dloss).check(out, grads, F32, "repeated")


@pytest.mark.parametrize("t,d,v", [(3, 65536, 70), (300, 65536, 40), (10, 20001, 300), (262144, 24, 900)])
def test_the_largest_widths_and_batches(handle, t, d, v):
    x, w, target, b, dloss = inputs(t, d, v, 1, True, 0.1)
    out, grads = run(handle, x, w, target, b, dloss, F32)
    Definition(x, w, target, b, dloss).check(out, grads, F32, f"{t} {d} {v}")


def test_more_than_the_largest_is_refused(handle):
    x, w, target, b, dloss = inputs(3, 8, 5, 1)
    big = torch.zeros(262145, 8, device="cuda", dtype=BF)
    with pytest.raises(ValueError, match="262144"):
        vocab.loss(handle, big, w, torch.zeros(262145, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="65536"):
        vocab.loss(handle, big.view(-1)[:65537].view(1, -1), torch.zeros(2, 65537, device="cuda", dtype=BF), target[:1])


def test_offsets_that_pass_32_bits(handle):
    """A matrix of 2.2e9 elements: the entries behind the 2^31st are where they belong, in z, in dx and in dw."""
    v, d, t = 540000, 4096, 6
    g = torch.Generator(device="cuda").manual_seed(3)
    w = torch.empty(v, d, device="cuda", dtype=BF)
    for i in range(0, v, 20000):
        w[i:i + 20000] = torch.randn(min(20000, v - i), d, device="cuda", generator=g) / 64.0
    x = torch.randn(t, d, device="cuda", generator=g).to(BF)
    target = torch.tensor([0, v - 1, v - 2, 524288, 524287, 100000], device="cuda")
    dloss = torch.ones(t, device="cuda") / t
    out = vocab.loss(handle, x, w, target)
    grads = vocab.loss_backward(handle, dloss, x, w, target, out.lse)
    z = torch.cat([x.double() @ w[i:i + 20000].double().T for i in range(0, v, 20000)], dim=1)
    lse = torch.logsumexp(z, 1)
    assert float((out.lse.double() - lse).abs().max()) <= 1e-4
    assert float((out.loss.double() - (lse - z.gather(1, target[:, None])[:, 0])).abs().max()) <= 1e-4
    p = torch.exp(z - lse[:, None])
    p.scatter_add_(1, target[:, None], -torch.ones(t, 1, device="cuda", dtype=torch.float64))
    p /= t
    dx = sum(p[:, i:i + 20000] @ w[i:i + 20000].double() for i in range(0, v, 20000))
    assert float((grads.dx.double() - dx).norm() / dx.norm()) <= 3 * UB
    for rows in (slice(0, 300), slice(524200, 524400), slice(v - 300, v)):
        want = p[:, rows].T @ x.double()
        assert float((grads.dw[rows].double() - want).norm() / want.norm()) <= 3 * UB


def test_two_handles_at_once():
    """Calls of two handles on two streams overlap and do not disturb one another."""
    a, b = stq.Handle(), stq.Handle()
    one, two = inputs(900, 300, 4000, 1, True, 0.2), inputs(400, 512, 7000, 2, False, 0.0)
    want = run(a, *one, F32), run(b, *two, BF)
    torch.cuda.synchronize()
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(8):
        with torch.cuda.stream(s[0]):
            got.append((0, run(a, *one, F32)))
        with torch.cuda.stream(s[1]):
            got.append((1, run(b, *two, BF)))
    torch.cuda.synchronize()
    for i, g in got:
        assert all(torch.equal(x, y) for p, q in zip(g, want[i]) for x, y in zip(p, q) if x is not None)
    a.close(), b.close()


@pytest.mark.parametrize("t,d", [(40, 300), (40, 1025), (300, 1025), (300, 4096)])
def test_a_gradient_does_not_go_by_which_others_are_asked_for(handle, t, d):
    """Sums of more than one part too; the vocabulary is one piece."""
    for dtype in (BF, F32):
        for bias in (True, False):
            x, w, target, b, dloss = inputs(t, d, 700, t + d, bias, 0.2)
            out, want = run(handle, x, w, target, b, dloss, dtype, want_dbias=True)
            for dx, dw, db in ((1, 1, 0), (1, 0, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)):
                g = vocab.loss_backward(handle, dloss, x, w, target, out.lse, bias=b, dtype=dtype, want_dx=bool(dx), want_dw=bool(dw),
                                        want_dbias=bool(db))
                for got, full, asked in zip(g, want, (dx, dw, db)):
                    assert (got is not None) == bool(asked) and (got is None or torch.equal(got, full)), (dtype, bias, dx, dw, db)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("d", [929, 4096])
@pytest.mark.parametrize("t", [3, 40, 700])
def test_gradients_of_confident_tokens(handle, t, d, bias):
    """Where the target has nearly all of the sum, p - 1 is much smaller than p, and what a logit is off by must not show in it: the loss
    and its gradients have to round a logit in the same way.  If they do, p_j is off by p_j times the others' shares times what their logits
    and its own are off by (what all are off by alike drops out), and by the roundings of lse and of z - lse, of exp and of the sum (24 U
    for the latter two)."""
    v, g = 32, torch.Generator(device="cuda").manual_seed(t + d)
    w = (torch.randn(v, d, device="cuda", generator=g) * (2 / d ** 0.5)).to(BF)
    target = torch.randint(0, v, (t,), device="cuda", generator=g)
    sure = 1 + 3 * torch.rand(t, 1, device="cuda", generator=g)
    x = (0.3 * torch.randn(t, d, device="cuda", generator=g) + sure * w[target].float()).to(BF)
    b = 0.5 * torch.randn(v, device="cuda", generator=g) if bias else None
    dloss = torch.full((t,), 1 / t, device="cuda")
    out = vocab.loss(handle, x, w, target, bias=b)
    x64, w64, b64 = x.double(), w.double(), 0.0 if b is None else b.double()
    z, a = x64 @ w64.T + b64, x64.abs() @ w64.abs().T + (0.0 if b is None else b64.abs())
    dz = 2 * U * (d / 16 + 2) * a + U * z.abs()
    lse, p = torch.logsumexp(z, 1, keepdim=True), torch.softmax(z, 1)
    hit = torch.nn.functional.one_hot(target, v).double()
    others = torch.softmax(z, 1).scatter(1, target[:, None], 0.0)
    grad = (p * (1 - hit) - hit * others.sum(1, keepdim=True)) / t
    apart = dz * (1 - p).clamp(min=0) + ((p * dz).sum(1, keepdim=True) - p * dz)
    sure_one = hit * (others * (dz + (hit * dz).sum(1, keepdim=True))).sum(1, keepdim=True)      # (1 - p without its cancellation)
    off = p / t * (torch.where(hit > 0, sure_one, apart) + U * (2 * lse.abs() + 4 * (z - lse).abs() + 24))
    rounded = UB * grad.abs() + off * (1 + UB)
    for dbias in (True, False):
        got = vocab.loss_backward(handle, dloss, x, w, target, out.lse, bias=b, want_dbias=dbias)
        want, tol = grad.T @ x64, rounded.T @ x64.abs() + 2 * U * (t / 16 + 34) * (grad.abs().T @ x64.abs())
        far = ((got.dw.double() - want).abs() / (tol * (1 + UB) + UB * want.abs() + 1e-44)).max()
        assert far <= 1, ("dw", dbias, float(far))
        want, tol = grad @ w64, rounded @ w64.abs() + 2 * U * (v / 16 + 64) * (grad.abs() @ w64.abs())
        far = ((got.dx.double() - want).abs() / (tol * (1 + UB) + UB * want.abs() + 1e-44)).max()
        assert far <= 1, ("dx", dbias, float(far))


@pytest.mark.parametrize("t,d,cuts", [(7000, 16, (1536, 4608, 6144)), (5000, 520, (3328,))])
def test_tokens_beside_the_ends_of_blocks(handle, t, d, cuts):
    """A loss of 600001 entries takes its tokens in blocks, so that its parts fit 256 MB: four parts of eight bytes to 128 entries up to 512
    columns, two beyond.  The tokens before and behind where blocks end."""
    x, w, target, b, dloss = inputs(t, d, 600001, 3, True, 0.3, sharp=1.0)
    out = vocab.loss(handle, x, w, target, bias=b)
    for at in cuts:
        rows = slice(at - 40, at + 40)
        Definition(x[rows], w, target[rows], b, dloss[rows]).check(vocab.LossOut(out.loss[rows], out.lse[rows]), None, BF, str(at))


@pytest.mark.parametrize("t,d,masked", [(200, 19000, 0.0), (1500, 6500, 0.2), (2500, 4000, 0.9)])
def test_many_columns(handle, t, d, masked):
    """Tiles of two blocks of rows for few tokens, and fewer rows than the plan counted on."""
    x, w, target, b, dloss = inputs(t, d, 500, t, True, masked)
    check = Definition(x, w, target, b, dloss)
    for dtype in (BF, F32):
        out, grads = run(handle, x, w, target, b, dloss, dtype)
        check.check(out, grads, dtype, f"{t} {d} {masked}")


@pytest.mark.parametrize("t", [1, 100, 129, 700])
def test_sums_leave_the_matrix_unit_in_parts(handle, t):
    """Sums of positive products, where all that is cut off is cut off to the same side: after each product of 16 terms up to one step, 2 U,
    of the sum so far, which begins anew after 512 terms (up to 128 tokens: 256), and a rounding for each part that is added.  (Whole
    sums lose 143 U of a logit: about 1.1 U of the sum so far, 256 times.)"""
    d, v, part = 4096, 300, 256 if t <= 128 else 512
    g = torch.Generator(device="cuda").manual_seed(t)
    x = (0.5 + torch.rand(t, d, device="cuda", generator=g)).to(BF)
    w = ((0.5 + torch.rand(v, d, device="cuda", generator=g)) * (20 / d)).to(BF)
    target = torch.randint(0, v, (t,), device="cuda", generator=g)
    out = vocab.loss(handle, x, w, target)
    z = x.double() @ w.double().T
    dz, total = torch.zeros_like(z), torch.zeros_like(z)
    for k in range(0, d, part):
        inner = torch.zeros_like(z)
        for i in range(k, k + part, 16):
            inner += x[:, i:i + 16].double() @ w[:, i:i + 16].double().T
            dz += 2 * U * inner
        total += inner
        dz += U * total
    lse = torch.logsumexp(z, 1)
    apart = (z - lse[:, None]).abs().amax(1)
    tol = dz.amax(1) + U * (2 * lse + 8 * apart + 2 * v / 128 + 64)
    far = (out.lse.double() - lse).abs()
    assert (tol < 45 * U * lse).all() and (far <= tol).all(), (float((far / tol).max()), float((far / U / lse).max()))


@pytest.mark.parametrize("t,d,v", [(5, 200, 333), (300, 200, 333), (300, 77, 1000), (700, 1025, 600)])
@pytest.mark.parametrize("extra,shift", [(8, 0), (0, 8), (3, 0), (1, 1), (0, 1)])
def test_results_of_any_pitch(handle, t, d, v, extra, shift):
    """dx and dw to rows with gaps, at any element: what lies between the rows and around them stays as it was."""
    x, w, target, b, dloss = inputs(t, d, v, 8, True, 0.2)
    lse = vocab.loss(handle, x, w, target, bias=b).lse
    for dtype, code in ((BF, stq.GRAD_BF16), (F32, stq.GRAD_F32)):
        want = vocab.loss_backward(handle, dloss, x, w, target, lse, bias=b, dtype=dtype)
        bufs = [torch.full((r * (d + extra) + shift + 64,), 7.0, device="cuda", dtype=k) for r, k in ((t, BF), (v, dtype))]
        dx, dw = (a[shift:shift + r * (d + extra)].view(r, d + extra) for a, r in zip(bufs, (t, v)))
        db = torch.empty(v, device="cuda")
        p = lambda t: t.data_ptr()      # noqa: E731
        rc = vocab._lib().stq_vocab_loss_backward(handle._h, p(dloss), p(x), d, p(w), d, p(b), p(target), IGNORE, p(lse), t, v, d, p(dx), d + extra,
                                                  p(dw), d + extra, code, p(db), torch.cuda.current_stream().cuda_stream)
        assert rc == 0 and torch.equal(db, want.dbias)
        for got, full, buf in ((dx, want.dx, bufs[0]), (dw, want.dw, bufs[1])):
            if got is dx or dtype == F32:
                assert torch.equal(got[:, :d], full)
            else:      # (rows off 16 bytes take tiles of one block, whose sums may be shared in another way: one step of bf16, or of the sum)
                assert ((got[:, :d].double() - full.double()).abs() <= 2 * UB * full.double().abs() + 2 * U * t * float(dloss.abs().max()) * 8).all()
            assert (got[:, d:] == 7.0).all() and (buf[:shift] == 7.0).all() and (buf[shift + got.numel():] == 7.0).all()
