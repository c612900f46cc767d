"""The norm of all gradients, its factor, and clipped gradients (stq_grad_norm, stq_grad_clip) against 64 bits.

Tolerances.  U = 2^-24 is half a step of fp32.  Up to 64 squares are summed in fp32, four sums of 16: a square and its place in the
sums see at most 1 + 16 + 2 roundings, all terms are positive, so a sum is off by 19 U of itself, its root by 10 U; the rounding of
the norm and the product with inv_scale add 2.  The factor has an addition, a division and a product more.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2604_06836_b200 import clip, stq   # noqa: E402
from paper_2604_06836_b200.optim import STQAdamW   # noqa: E402

BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U = 2.0 ** -24

NORM, FACTOR = 12 * U, 15 * U


@pytest.fixture(scope="module")
def handle():
    h = stq.Handle()
    yield h
    h.device_status()
    h.close()


def many(lengths, dtypes, seed=0, scale=1e-2):
    """Gradients of these lengths, some of them views that begin in the middle of a buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(lengths):
        x = torch.randn(n + 9, device="cuda", generator=g) * (scale * 10.0 ** (i % 4 - 2))
        out.append(x.to(dtypes[i % len(dtypes)])[i % 9:i % 9 + n])
    return out


def exact(grads, max_norm=math.inf, inv=1.0, eps=1e-6):
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads)) * inv
    return norm, inv * min(1.0, max_norm / (norm + eps) if norm < math.inf else 0.0)


def near(got, want, rel):
    assert abs(float(got) - want) <= rel * abs(want), (float(got), want)


LENGTHS = [1, 7, 8, 255, 4096, 65536, 100003, 3, 16384, 1 << 20]


@pytest.mark.parametrize("dtypes", [[F32], [BF], [F16], [F32, BF, F16]])
def test_norm_and_clip(handle, dtypes):
    for inv in (None, torch.full((1,), 1 / 64, device="cuda")):
        grads = many(LENGTHS, dtypes)
        scale = 1.0 if inv is None else 1 / 64
        norm, factor = exact(grads, 0.25, scale)
        r = clip.grad_norm(handle, grads, max_norm=0.25, inv_scale=inv)
        near(r.norm, norm, NORM)
        near(r.factor, factor, FACTOR)
        again = clip.grad_norm(handle, grads, max_norm=0.25, inv_scale=inv)
        assert torch.equal(r.norm, again.norm)
        near(clip.grad_norm(handle, grads, inv_scale=inv).factor, scale, 0)
        for odt in (None, F32):
            out = [torch.full_like(g, 7.0, dtype=odt) for g in grads]
            before = [g.clone() for g in grads]
            c = clip.clip_grads(handle, grads, 0.25, inv_scale=inv, out=out)
            assert torch.equal(c.norm, r.norm) and torch.equal(c.factor, r.factor)
            for g, b, o in zip(grads, before, out):
                assert torch.equal(g, b)
                assert torch.equal(o, (g.float() * r.factor).to(o.dtype))      # one product, rounded once
        inside = [torch.cat([g, g[:1]])[:-1] for g in grads]
        clip.clip_grads(handle, inside, 0.25, inv_scale=inv)
        for g, i in zip(grads, inside):
            assert torch.equal(i, (g.float() * r.factor).to(g.dtype))


def test_what_lies_between_the_tensors_stays(handle):
    buf = torch.full((10000,), 3.0, device="cuda")
    views = [buf[5:17], buf[20:21], buf[33:5000], buf[5001:9998]]
    for v in views:
        v.normal_()
    mask = torch.ones(10000, dtype=torch.bool, device="cuda")
    for a, b in ((5, 17), (20, 21), (33, 5000), (5001, 9998)):
        mask[a:b] = False
    want = [v * clip.grad_norm(handle, views, max_norm=1.0).factor for v in views]
    clip.clip_grads(handle, views, 1.0)
    assert (buf[mask] == 3.0).all()
    assert all(torch.equal(v, w) for v, w in zip(views, want))


def test_values_whose_squares_leave_the_range(handle):
    big = torch.randn(5000, device="cuda") * 1e30
    small = torch.randn(5000, device="cuda") * 1e-30
    for grads in ([big], [small], [big, small], [small, torch.zeros(100000, device="cuda")], [big.to(BF)], [small.to(BF)]):
        r = clip.grad_norm(handle, grads, max_norm=1.0)
        near(r.norm, exact(grads)[0], NORM)
    one = torch.full((1,), 3e-45, device="cuda")
    assert float(clip.grad_norm(handle, [one]).norm) == float(one)


def test_nothing_to_sum(handle):
    inv = torch.full((1,), 0.5, device="cuda")
    for grads in ([], [None], [torch.zeros(0, device="cuda")], [torch.zeros(1000, device="cuda", dtype=BF)]):
        r = clip.clip_grads(handle, grads, 1.0, inv_scale=inv)
        assert float(r.norm) == 0.0 and float(r.factor) == 0.5


@pytest.mark.parametrize("dtype", [F32, BF, F16])
def test_infinities_and_nan(handle, dtype):
    for value in (math.inf, -math.inf, math.nan):
        for at in (0, 12344):
            g = torch.ones(12345, device="cuda", dtype=dtype)
            g[at] = value
            flag = torch.zeros(1, device="cuda")
            r = clip.grad_norm(handle, [g[:100] * 0 + 1, g], max_norm=1.0, found_inf=flag)
            if at == 0:      # the first tensor holds value * 0 + 1, which is NaN
                norm = factor = math.nan
            else:
                norm, factor = (math.nan, math.nan) if math.isnan(value) else (math.inf, 0.0)
            assert str(float(r.norm)) == str(norm) and str(float(r.factor)) == str(factor) and float(flag) == 1.0
    flag = torch.zeros(1, device="cuda")
    clip.grad_norm(handle, [torch.ones(10, device="cuda", dtype=dtype)], max_norm=1.0, found_inf=flag)
    assert float(flag) == 0.0


def test_more_tensors_than_one_launch_takes(handle):
    grads = many([1 + i % 700 for i in range(2500)], [F32, BF])
    norm, factor = exact(grads, 0.5)
    before = handle.launch_count
    r = clip.clip_grads(handle, grads, 0.5, out=(out := [torch.empty_like(g) for g in grads]))
    assert handle.launch_count - before == 6
    near(r.norm, norm, NORM)
    assert all(torch.equal(o, (g.float() * r.factor).to(g.dtype)) for g, o in zip(grads, out))


def test_layouts(handle):
    g = torch.randn(64, 33, device="cuda")
    t = torch.empty_strided((64, 33), (1, 64), device="cuda").copy_(g)
    assert torch.equal(clip.grad_norm(handle, [g]).norm.round(decimals=3), clip.grad_norm(handle, [t]).norm.round(decimals=3))
    clip.clip_grads(handle, [t], 1.0)
    near(t.double().norm(), 1.0, 1e-5)
    for bad in (g[:, :5], g[::2], g[:, :1].expand(64, 4)):
        with pytest.raises(ValueError, match="dense"):
            clip.grad_norm(handle, [bad])


def test_refusals(handle):
    g, h = torch.ones(100, device="cuda"), torch.ones(200, device="cuda")
    with pytest.raises(stq.StqError) as e:      # written twice
        clip.clip_grads(handle, [g, g], 1.0)
    assert e.value.code == -5
    with pytest.raises(stq.StqError) as e:      # a result where another gradient lies
        clip.clip_grads(handle, [h[:100], h[100:]], 1.0, out=[h[50:150], torch.empty(100, device="cuda")])
    assert e.value.code == -5
    assert (g == 1).all() and (h == 1).all()
    for kw in ({"max_norm": 0.0}, {"max_norm": -1.0}, {"max_norm": math.nan}, {"max_norm": 1.0, "eps": -1.0}):
        with pytest.raises(ValueError):
            clip.grad_norm(handle, [g], **kw)
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        clip.grad_norm(handle, [g.double()])
    with pytest.raises(ValueError, match="device"):
        clip.grad_norm(handle, [g.cpu()])
    with pytest.raises(ValueError, match="type of its gradient"):
        clip.clip_grads(handle, [g], 1.0, out=[g.to(BF)])
    with pytest.raises(ValueError, match="layout"):
        clip.clip_grads(handle, [g], 1.0, out=[h])


def test_a_captured_call_replays_on_new_values(handle):
    grads = many([1000, 70001], [F32])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        clip.clip_grads(handle, grads, 0.1)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = clip.clip_grads(handle, grads, 0.1)
    for seed in (1, 2):
        new = many([1000, 70001], [F32], seed)
        for g, n in zip(grads, new):
            g.copy_(n)
        graph.replay()
        near(r.norm, exact(new)[0], NORM)
        f = float(r.factor)
        assert all(torch.equal(g, n * f) for g, n in zip(grads, new))


def test_on_another_stream(handle):
    s = torch.cuda.Stream()
    g = torch.zeros(1 << 24, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(2000000)
        g.fill_(2.0)
    r = clip.grad_norm(handle, [g], stream=s)
    torch.cuda.current_stream().wait_stream(s)
    near(r.norm, 2.0 * 4096, NORM)


def test_generators(handle):
    """A generator is gone through once, also where its tensors are needed twice (on another stream, counted as changed)."""
    g = [torch.full((100,), 2.0, device="cuda"), None, torch.full((300,), 2.0, device="cuda")]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (None, s):
        near(clip.grad_norm(handle, (t for t in g), stream=stream).norm, 40.0, NORM)
        out = [None if t is None else torch.empty_like(t) for t in g]
        before = [(t._version, o._version) for t, o in zip(g, out) if t is not None]
        clip.clip_grads(handle, iter(g), 20.0, out=iter(out), stream=stream)
        torch.cuda.current_stream().wait_stream(s)
        assert [(t._version, o._version) for t, o in zip(g, out) if t is not None] == [(a, b + 1) for a, b in before]
        assert all(torch.allclose(o, t * 0.5) for t, o in zip(g, out) if t is not None)
    clip.clip_grads(handle, (t for t in g), 20.0, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.allclose(t, torch.ones_like(t)) for t in g if t is not None)


def parameters(seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.nn.Parameter(torch.randn(n, device="cuda", generator=g)) for n in (4096, 1000, 13, 70000)]


@pytest.mark.parametrize("scaled", [False, True])
def test_the_optimizer_clips_as_it_steps(scaled):
    """The step multiplies each gradient with the factor, rounded once: the same numbers as a gradient clipped in place."""
    ours, plain = parameters(), parameters()
    a = STQAdamW(ours, lr=1e-2, policy="fixed", init_bits=8, max_norm=0.5)
    b = STQAdamW(plain, lr=1e-2, policy="fixed", init_bits=8)
    inv = torch.full((1,), 1 / 128, device="cuda") if scaled else None
    a.grad_scaler_inv = inv
    for t in range(8):
        for p, q in zip(ours, plain):
            p.grad = torch.randn_like(p) * (0.001 if t % 3 == 0 else 0.1) * (128.0 if scaled else 1.0)
            q.grad = p.grad.clone()
        want = math.sqrt(sum(float(p.grad.double().square().sum()) for p in ours)) / (128 if scaled else 1)
        kept = [p.grad.clone() for p in ours]
        clip.clip_grads(b.handle, [q.grad for q in plain], 0.5, inv_scale=inv)
        a.step(), b.step()
        near(a.last_norm, want, NORM)
        assert all(torch.equal(p.grad, k) for p, k in zip(ours, kept))
        assert all(torch.equal(p, q) for p, q in zip(ours, plain)), t


@pytest.mark.parametrize("order", ["paper", "fused"])
def test_the_policy_sees_clipped_gradients(order):
    """Widths under gradients that are clipped are those under gradients that arrive clipped."""
    ours, plain = parameters(), parameters()
    a = STQAdamW(ours, lr=1e-2, max_norm=0.5, interval=5, order=order)
    b = STQAdamW(plain, lr=1e-2, interval=5, order=order)
    for t in range(12):
        for k, (p, q) in enumerate(zip(ours, plain)):
            p.grad = torch.randn_like(p) * 10.0 ** (k - 2)
            q.grad = p.grad.clone()
        clip.clip_grads(b.handle, [q.grad for q in plain], 0.5)
        a.step(), b.step()
        assert (a.bits_m == b.bits_m).all()


def test_a_step_with_a_norm_that_is_not_finite_is_left_out():
    ps = parameters()
    opt = STQAdamW(ps, lr=1e-2, policy="fixed", init_bits=8, max_norm=1.0)
    opt.found_inf = torch.zeros(1, device="cuda")
    before = [p.detach().clone() for p in ps]
    for p in ps:
        p.grad = torch.ones_like(p)
    ps[1].grad[3] = math.inf
    opt.step()
    assert opt.t == 0 and opt.skipped_steps == 1 and all(torch.equal(p, b) for p, b in zip(ps, before))
    opt.found_inf.zero_()
    ps[1].grad[3] = 1.0
    opt.step()
    assert opt.t == 1 and not torch.equal(ps[0], before[0])
    with pytest.raises(ValueError, match="max_norm"):
        STQAdamW(ps, max_norm=0.0)


def test_a_tensor_of_more_than_32_bits_of_elements(handle):
    n = (1 << 31) + 12345
    g = torch.zeros(n, device="cuda", dtype=BF)
    g[-5:] = 3.0
    g[:4] = 1.0
    r = clip.grad_norm(handle, [g], max_norm=0.5)
    near(r.norm, 7.0, NORM)
    clip.clip_grads(handle, [g], 3.5)      # factor 1 / 2, up to eps
    assert g[-5:].tolist() == [1.5] * 5 and g[:4].tolist() == [0.5] * 4 and float(g[n // 2].float()) == 0.0


def test_two_handles_at_once():
    a, b = stq.Handle(), stq.Handle()
    one, two = many([1 << 22, 777], [F32], 1), many([1 << 20] * 300, [BF], 2)
    want = clip.grad_norm(a, one).norm, clip.grad_norm(b, two).norm
    torch.cuda.synchronize()
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(10):
        got.append((0, clip.grad_norm(a, one, stream=s[0]).norm))
        got.append((1, clip.grad_norm(b, two, stream=s[1]).norm))
    torch.cuda.synchronize()
    assert all(torch.equal(n, want[i]) for i, n in got)
    a.close(), b.close()


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("scaled", [False, True])
def test_a_step_that_is_left_out_does_not_hold_up_the_next(bad, scaled):
    """found_inf belongs to the caller: the optimizer reads it and leaves it as it is, also where it is set once for all steps."""
    ps = parameters()
    opt = STQAdamW(ps, lr=1e-2, policy="fixed", init_bits=8, max_norm=1.0)
    opt.found_inf = torch.zeros(1, device="cuda")
    opt.grad_scaler_inv = torch.full((1,), 1 / 128, device="cuda") if scaled else None
    taken = 0
    for t, value in enumerate((1.0, bad, 1.0, 1.0, bad, bad, 1.0)):
        for p in ps:
            p.grad = torch.ones_like(p)
        ps[1].grad[3] = value
        before = ps[0].detach().clone()
        opt.step()
        taken += value == 1.0
        assert (opt.t, opt.skipped_steps) == (taken, t + 1 - taken)
        assert torch.equal(ps[0], before) == (value != 1.0) and float(opt.found_inf) == 0.0
    opt.found_inf.fill_(1.0)      # what the caller found
    opt.step()
    assert opt.t == taken and float(opt.found_inf) == 1.0


def test_scalars_lie_in_places_of_their_own(handle):
    """A factor or a flag inside of what is scaled would be written while it is read: refused, and nothing is changed."""
    g, out = torch.full((64,), 3.0, device="cuda"), torch.zeros(64, device="cuda")
    one, two = out.new_zeros(1), out.new_zeros(1)
    L, p = clip._lib(), lambda t: t.data_ptr()      # noqa: E731
    def call(fn, to, norm, factor, flag):      # noqa: E306
        rows, n = clip._lists.rows([g], None if to is None else [to], 0)
        return fn(handle._h, rows, n, None, 1.0, 1e-6, p(norm), p(factor), None if flag is None else p(flag), None)
    for to in (None, out):      # in place, and elsewhere
        for inside in [g[5:6], g[63:]] + ([] if to is None else [out[:1], out[63:]]):
            for scalars in ((inside, one, None), (one, inside, None), (one, two, inside)):
                assert call(L.stq_grad_clip, to, *scalars) == -5
    for scalars in ((one, one, None), (one, two, one), (one, two, two)):
        assert call(L.stq_grad_clip, out, *scalars) == -5 and call(L.stq_grad_norm, None, *scalars) == -5
    torch.cuda.synchronize()
    assert (g == 3.0).all() and (out == 0.0).all() and float(one) == float(two) == 0.0
    assert call(L.stq_grad_clip, out[:64], one, two, None) == 0      # (side by side is fine)
    assert call(L.stq_grad_norm, None, g[5:6], g[6:7], None) == 0      # (a norm reads its gradients once, before it writes)
    with pytest.raises(stq.StqError) as e:
        clip.clip_grads(handle, [g], 1.0, found_inf=g[2:3])
    assert e.value.code == -5
