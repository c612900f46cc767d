"""The 8-bit operators (stq_q8_*) against their formulas in 64 bits, element by element.

Tolerances come from the number formats: 2^-24 relative for an fp32 operation, 2^-8 for a rounding to bf16, and for a
sum the bound is taken relative to the sum of the terms' magnitudes.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2604_06836_b200 import q8, stq   # noqa: E402

BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-6
U = 2.0 ** -24          # half an ulp of fp32
UB = 2.0 ** -8           # half an ulp of bf16 (8 significant bits)


@pytest.fixture(scope="module")
def handle():
    h = stq.Handle()
    yield h
    h.device_status()
    h.close()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def hidden(rows, cols, seed, dtype=F32, scale=1.0):
    g = gen(seed)
    x = torch.randn(rows, cols, device="cuda", generator=g) * torch.exp(0.7 * torch.randn(cols, device="cuda", generator=g))
    if rows > 3:
        x[2] = 0.0                      # a padding token
    return (x * scale).to(dtype)


def pitched(x, extra, shift=0):
    """The same matrix with `extra` more elements to a row, beginning `shift` elements into the buffer."""
    r, c = x.shape
    buf = torch.full((r * (c + extra) + shift + 64,), 7.0, device=x.device, dtype=torch.float32).to(x.dtype)
    v = buf[shift:shift + r * (c + extra)].view(r, c + extra)[:, :c]
    v.copy_(x)
    return v


def check_rows(rows, want, near, rel, what):
    """8-bit rows against the exact values `want` (float64): the scale to `rel`, the codes equal except where the exact
    quotient lies within `near` of a rounding boundary."""
    top = want.abs().amax(1)
    scale = rows.scale.double()
    zero = top < 2.0 ** -100
    assert (scale[zero] == 0).all() and (rows.q[zero] == 0).all(), what
    assert ((scale - top / 127).abs() <= rel * top / 127).all(), what
    quot = want * torch.where(zero, 0.0, 127.0 / torch.where(zero, 1.0, top))[:, None]
    off = (rows.q.double() - quot).abs()
    assert (off <= 0.5 + near).all(), (what, float(off.max()))


def check_values(out, rows, what):
    want = (rows.q.float() * rows.scale[:, None]).to(BF)
    assert torch.equal(torch.nan_to_num(out, nan=1e30), torch.nan_to_num(want, nan=1e30)), what


COLS = [1, 2, 7, 8, 64, 127, 128, 129, 255, 257, 768, 1601, 2050, 4096, 8208, 9001, 16640]


# ---- rows ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("cols", COLS)
def test_quantize_rows(handle, cols, dtype):
    x = hidden(5, cols, cols, dtype, 0.02)
    r = q8.quantize_rows(handle, x)
    assert r.q.stride(0) % 16 == 0 and r.q.shape == x.shape
    check_rows(r, x.double(), 127 * 3 * U, 2 * U, f"rows {cols}")
    # the same values through other pitches and offsets give the same codes
    for extra, shift in ((3, 0), (2, 2), (8, 8), (8, 1)):
        r2 = q8.quantize_rows(handle, pitched(x, extra, shift))
        assert torch.equal(r.q, r2.q) and torch.equal(r.scale, r2.scale)


def test_rows_that_hold_what_a_code_cannot(handle):
    x = hidden(7, 300, 1)
    x[0, 17] = float("inf")
    x[1, 299] = float("nan")
    x[3] = 1e-35                         # below the smallest scale
    x[4] = 3.0e38
    x[5] = -0.0
    for t in (x, x.to(BF), x[:, :299], pitched(x, 8)):
        r = q8.quantize_rows(handle, t)
        assert torch.isnan(r.scale[0]) and (r.q[0] == 0).all()
        if t.shape[1] == 300:
            assert torch.isnan(r.scale[1]) and (r.q[1] == 0).all()
        assert (r.scale[[2, 3, 5]] == 0).all() and (r.q[[2, 3, 5]] == 0).all()
        assert torch.isfinite(r.scale[4]) and (r.q[4] == 127).all()
        assert int(r.q[6].abs().max()) == 127


# ---- norm ------------------------------------------------------------------------------------------------------
def norm_exact(x, res, w):
    h = x.double() + (0 if res is None else res.double())
    rstd = (h.square().mean(1) + EPS).rsqrt()
    return h, rstd, h * rstd[:, None] * w.double()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows", [1, 6])
@pytest.mark.parametrize("cols", COLS)
def test_norm(handle, cols, rows, dtype):
    x, res = hidden(rows, cols, 10 + cols, dtype), hidden(rows, cols, 20 + cols, dtype, 2.0)
    w = 1 + 0.1 * torch.randn(cols, device="cuda", generator=gen(3))
    for r in (res, None):
        out = q8.norm(handle, x, w, residual=r, eps=EPS, values=True)
        h, rstd, y = norm_exact(x, r, w)
        if r is None:
            assert out.h is x
        else:
            assert torch.equal(out.h, (x.float() + r.float()).to(dtype))
        # the mean is a tree of fp32 sums of at most 8 * (cols / 256 + 1) and log2 steps of squares, all positive
        assert ((out.rstd.double() - rstd).abs() <= 40 * U * rstd).all()
        check_rows(out.rows, y, 127 * 5 * U, 48 * U, f"norm {rows}x{cols}")
        check_values(out.values, out.rows, "norm values")
        out2 = q8.norm(handle, pitched(x, 8, 8), w, residual=None if r is None else pitched(r, 5, 1), eps=EPS)
        assert out2.values is None
        assert torch.equal(out2.rows.q, out.rows.q) and ((out2.rows.scale - out.rows.scale).abs() <= 48 * U * out.rows.scale).all()


def test_norm_of_rows_that_are_not_finite(handle):
    x = hidden(4, 512, 5)
    x[0, 3], x[1, 4] = float("nan"), float("-inf")
    out = q8.norm(handle, x, torch.ones(512, device="cuda"))
    assert torch.isnan(out.rows.scale[:2]).all() and (out.rows.q[:2] == 0).all()
    assert (out.rows.scale[2] == 0) and torch.isfinite(out.rows.scale[3])


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 1600), (3, 129), (37, 64), (700, 257), (5, 2048), (9, 2304), (300, 1277),
                                       (6, 8192), (4, 16384), (7, 16400), (3, 20001), (2, 49152)])
def test_norm_backward(handle, rows, cols, dtype):
    h = hidden(rows, cols, rows + cols, dtype, 2.0)
    g = gen(7)
    w = 1 + 0.1 * torch.randn(cols, device="cuda", generator=g)
    dy = (1e-3 * torch.randn(rows, cols, device="cuda", generator=g)).to(dtype)
    dres = (1e-3 * torch.randn(rows, cols, device="cuda", generator=g)).to(dtype)
    rstd = (h.double().square().mean(1) + EPS).rsqrt().float()
    for r in (dres, None):
        dx, dw = q8.norm_backward(handle, dy, h, w, rstd, dres=r)
        rs = rstd.double()[:, None]
        xh, up = h.double() * rs, dy.double() * w.double()
        c = (up * xh).mean(1, keepdim=True)
        want = rs * (up - xh * c) + (0 if r is None else r.double())
        size = rs * (up.abs() + xh.abs() * (up * xh).abs().mean(1, keepdim=True)) + (0 if r is None else r.double().abs())
        tol = 64 * U * size + (UB * 1.01 * want.abs() if dtype == BF else 0)
        assert ((dx.double() - want).abs() <= tol).all(), float(((dx.double() - want).abs() - tol).max())
        wantw, sizew = (dy.double() * xh).sum(0), (dy.double() * xh).abs().sum(0)
        assert ((dw.double() - wantw).abs() <= 64 * U * sizew).all()
    dx2, dw2 = q8.norm_backward(handle, pitched(dy, 1), pitched(h, 8), w, rstd)
    assert torch.allclose(dx2.float(), dx.float(), rtol=UB if dtype == BF else 1e-4, atol=1e-6 * float(dx.float().abs().max()))
    assert torch.allclose(dw2, dw, rtol=1e-4, atol=1e-5 * float(dw.abs().max()))
    again = q8.norm_backward(handle, dy, h, w, rstd)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)      # no order of sums that changes


def test_norm_backward_against_differences(handle):
    """Directional differences of sum(y * v) + sum(h * u) in 64 bits against the kernel's gradients."""
    g = gen(11)
    rows, cols = 9, 200
    x = torch.randn(rows, cols, device="cuda", generator=g)
    w = 1 + 0.1 * torch.randn(cols, device="cuda", generator=g)
    v, u = (torch.randn(rows, cols, device="cuda", generator=g) for _ in range(2))
    f = lambda a, b: float((norm_exact(a, None, b)[2] * v.double()).sum() + (a.double() * u.double()).sum())  # noqa: E731
    out = q8.norm(handle, x, w, eps=EPS)
    dx, dw = q8.norm_backward(handle, v, out.h, w, out.rstd, dres=u)
    for seed in range(3):
        d, e = torch.randn(rows, cols, device="cuda", generator=gen(seed)).double(), torch.randn(cols, device="cuda", generator=gen(9 + seed)).double()
        s = 1e-6
        num = (f(x.double() + s * d, w.double() + s * e) - f(x.double() - s * d, w.double() - s * e)) / (2 * s)
        ana = float((dx.double() * d).sum() + (dw.double() * e).sum())
        assert abs(num - ana) <= 1e-4 * float((dx.double() * d).abs().sum())


# ---- activations ---------------------------------------------------------------------------------------------------
def act_exact(z, kind):
    z = z.double()
    if kind == "silu_gated":
        f = z.shape[1] // 2
        return z[:, :f] * torch.sigmoid(z[:, :f]) * z[:, f:]
    return torch.nn.functional.gelu(z, approximate="tanh")


def act_grad_exact(z, da, kind):
    z = z.double().requires_grad_(True)
    act_exact(z, kind).backward(da.double())
    return z.grad


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("kind", ["silu_gated", "gelu"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 6400), (5, 2), (6, 127), (6, 128), (6, 130), (4, 264), (33, 1000), (5, 5121),
                                       (4, 8208), (3, 16384), (2, 16640), (2, 17001)])
def test_act_and_its_backward(handle, rows, cols, kind, dtype):
    parts = 2 if kind == "silu_gated" else 1
    z = hidden(rows, parts * cols, cols + parts, dtype)
    out = q8.act(handle, z, kind, checkpoint=True, values=True)
    # fp32 exp and divide: the exponent's argument is rounded, |z| up to ~20 here
    check_rows(out.rows, act_exact(z, kind), 127 * 1e-5, 1e-5, f"{kind} {rows}x{cols}")
    check_values(out.values, out.rows, "act values")
    plain = q8.act(handle, z, kind)
    assert plain.checkpoint is None and torch.equal(plain.rows.q, out.rows.q) and torch.equal(plain.rows.scale, out.rows.scale)
    ck = out.checkpoint
    zp = z.double().reshape(rows, parts, cols)
    pad = -cols % 128
    full = torch.nn.functional.pad(zp, (0, pad)).reshape(rows, parts, -1, 128)
    top = full.abs().amax(3)
    assert ((ck.scale.double() - top / 127).abs() <= 2 * U * top / 127).all()
    quot = full * torch.where(top == 0, 0.0, 127.0 / torch.where(top == 0, 1.0, top))[..., None]
    got = torch.nn.functional.pad(ck.q[:, :, :cols].double(), (0, pad)).reshape(full.shape)
    assert ((got - quot).abs() <= 0.5 + 127 * 3 * U).all()
    # decoded once more by the backward pass
    da = (1e-3 * torch.randn(rows, cols, device="cuda", generator=gen(4))).to(dtype)
    dz = q8.act_backward(handle, da, ck)
    kept = ck.values()
    want = act_grad_exact(kept, da, kind)
    other = kept.double()[:, cols:].repeat(1, 2).abs() if parts == 2 else 0
    size = da.double().abs().repeat(1, parts) * (1 + kept.double().abs()) * (1 + other)
    tol = 1e-5 * size + (1.01 * UB * want.abs() if dtype == BF else 0)
    assert ((dz.double() - want).abs() <= tol).all(), float(((dz.double() - want).abs() / size).max())
    zs, das = pitched(z, 3, 1), pitched(da, 8, 8)
    o2 = q8.act(handle, zs, kind, checkpoint=True)
    assert torch.equal(o2.rows.q, out.rows.q) and torch.equal(o2.checkpoint.scale, ck.scale)
    assert torch.equal(o2.checkpoint.q[:, :, :cols], ck.q[:, :, :cols])
    assert torch.equal(q8.act_backward(handle, das, o2.checkpoint), dz)


def test_act_where_the_input_is_extreme(handle):
    """Large magnitudes saturate, an infinity poisons its row and its block and nothing else."""
    z = hidden(3, 512, 8)
    z[0, :4] = torch.tensor([90.0, -90.0, 1e4, -1e4], device="cuda")
    out = q8.act(handle, z, "silu_gated", checkpoint=True)
    check_rows(out.rows, act_exact(z, "silu_gated"), 127 * 1e-5, 1e-5, "extreme")
    z[1, 130] = float("inf")
    out = q8.act(handle, z, "gelu", checkpoint=True, values=True)
    assert torch.isnan(out.rows.scale[1]) and torch.isfinite(out.rows.scale[[0, 2]]).all()
    assert torch.isnan(out.values[1].float()).all() and not torch.isnan(out.values[[0, 2]].float()).any()
    bad = torch.isnan(out.checkpoint.scale[:, 0])
    assert bad[1, 1] and int(bad.sum()) == 1
    dz = q8.act_backward(handle, torch.ones(3, 512, device="cuda"), out.checkpoint)
    assert torch.isnan(dz[1, 128:256]).all() and int(torch.isnan(dz).sum()) == 128


def test_act_backward_against_differences(handle):
    for kind, parts in (("silu_gated", 2), ("gelu", 1)):
        g = gen(13)
        z = torch.randn(7, parts * 130, device="cuda", generator=g)
        v = torch.randn(7, 130, device="cuda", generator=g)
        ck = q8.act(handle, z, kind, checkpoint=True).checkpoint
        at = ck.values().double()
        dz = q8.act_backward(handle, v, ck).double()
        d = torch.randn(7, parts * 130, device="cuda", generator=g).double()
        s = 1e-6
        num = float(((act_exact(at + s * d, kind) - act_exact(at - s * d, kind)) * v.double()).sum()) / (2 * s)
        assert abs(num - float((dz * d).sum())) <= 1e-4 * float((dz * d).abs().sum())


# ---- products ------------------------------------------------------------------------------------------------------
def codes(rows, cols, seed, scale=1.0):
    g = gen(seed)
    r = q8.alloc_rows(rows, cols, "cuda")
    r.q.copy_(torch.randint(-127, 128, (rows, cols), device="cuda", generator=g, dtype=torch.int32).to(torch.int8))
    r.scale.copy_(scale * torch.rand(rows, device="cuda", generator=g) + 1e-3 * scale)
    if rows > 4:
        r.q[3] = 0
        r.scale[3] = 0.0
    return r


def dec(r):
    return r.q.double() * r.scale.double()[:, None]


def near(got, want, size, dtype, rel):
    tol = rel * size + (1.01 * UB * want.abs() if dtype == BF else 0)
    err = (got.double() - want).abs()
    assert (err <= tol).all(), float((err / size.clamp_min(1e-300)).max())


SIZES = [(1, 1, 1), (1, 8, 16), (1, 1600, 768), (2, 65, 33), (3, 257, 128), (16, 640, 512), (17, 130, 769), (33, 1283, 100),
         (64, 96, 2050), (65, 256, 256), (127, 129, 127), (128, 128, 128), (129, 300, 640), (197, 2304, 768), (256, 512, 1024),
         (300, 77, 1601), (513, 1000, 264), (1003, 1283, 769), (2100, 264, 640)]


@pytest.mark.parametrize("t,n,k", SIZES)
def test_linear(handle, t, n, k):
    x, w = codes(t, k, 1 + t, 0.05), codes(n, k, 2 + n, 0.002)
    b = 0.1 * torch.randn(n, device="cuda", generator=gen(3))
    want = dec(x) @ dec(w).T
    for dtype in (F32, BF):
        for bias in (None, b):
            ref = want if bias is None else want + bias.double()
            got = q8.linear(handle, x, w, bias=bias, dtype=dtype)
            assert got.shape == (t, n) and got.dtype == dtype
            # the integer sum is exact: one conversion, two products, one addition
            near(got, ref, want.abs() + b.double().abs() + 1e-300, dtype, 4 * U)


@pytest.mark.parametrize("t,n,k", SIZES)
def test_linear_backward(handle, t, n, k):
    x, w = codes(t, k, 1 + t, 0.05), codes(n, k, 2 + n, 0.002)
    dy = (1e-3 * torch.randn(t, n, device="cuda", generator=gen(5))).to(BF)
    dx, dw = dy.double() @ dec(w), dy.double().T @ dec(x)
    sx, sw = dy.double().abs() @ dec(w).abs(), dy.double().abs().T @ dec(x).abs()
    for dtype, rel in ((F32, 2.0 ** -17 + 2.0 ** -18), (BF, UB + 2.0 ** -17)):
        near(q8.linear_dx(handle, dy, w, dtype=dtype), dx, sx + 1e-300, dtype, rel)
        near(q8.linear_dw(handle, dy, x, dtype=dtype), dw, sw + 1e-300, dtype, rel)
    db = q8.bias_grad(handle, dy)
    near(db, dy.double().sum(0), dy.double().abs().sum(0) + 1e-300, F32, 64 * U)
    assert torch.equal(db, q8.bias_grad(handle, dy))
    a, b = q8.linear_dw(handle, dy, x, dtype=F32), q8.linear_dx(handle, dy, w, dtype=F32)
    assert torch.equal(a, q8.linear_dw(handle, dy, x, dtype=F32)) and torch.equal(b, q8.linear_dx(handle, dy, w, dtype=F32))
    # a gradient that is a slice of a wider one, on any offset
    for extra, shift in ((1, 0), (8, 8), (6, 3)):
        dys = pitched(dy, extra, shift)
        assert torch.equal(a, q8.linear_dw(handle, dys, x, dtype=F32)) and torch.equal(b, q8.linear_dx(handle, dys, w, dtype=F32))
        assert torch.allclose(db, q8.bias_grad(handle, dys), rtol=0, atol=float(64 * U * dy.double().abs().sum(0).max()))


@pytest.mark.parametrize("t,n,k,dtype", [(8200, 1608, 1603, BF), (8200, 1607, 1600, BF), (4100, 1608, 2056, F32), (1601, 8208, 1600, BF)])
def test_linear_backward_of_a_batch(handle, t, n, k, dtype):
    """Large results: for a bf16 one the 8-bit operand is converted ahead of the product, one launch more."""
    x, w = codes(t, k, 1 + t, 0.05), codes(n, k, 2 + n, 0.002)
    dy = (1e-3 * torch.randn(t, n, device="cuda", generator=gen(5))).to(BF)
    rel = UB + 2.0 ** -17 if dtype == BF else 2.0 ** -17
    before = handle.launch_count
    dx = q8.linear_dx(handle, dy, w, dtype=dtype)
    middle = handle.launch_count
    dw = q8.linear_dw(handle, dy, x, dtype=dtype)
    assert dtype == F32 or max(middle - before, handle.launch_count - middle) >= 2
    near(dx, dy.double() @ dec(w), dy.double().abs() @ dec(w).abs() + 1e-300, dtype, rel)
    near(dw, dy.double().T @ dec(x), dy.double().abs().T @ dec(x).abs() + 1e-300, dtype, rel)
    w.scale[n - 1] = float("nan")
    w.q[n - 1] = 0
    assert torch.isnan(q8.linear_dx(handle, dy, w, dtype=dtype)).all()
    x.scale[t - 1] = float("nan")
    x.q[t - 1] = 0
    assert torch.isnan(q8.linear_dw(handle, dy, x, dtype=dtype)).all()


@pytest.mark.parametrize("depth", [1003, 20000])
def test_fp32_gradients_of_long_sums(handle, depth):
    """Random signs: the result is far smaller than the terms' sum, and a bias of the sums would show.  At most 16 steps of
    the matrix unit at full size go into a partial sum before it is added up in fp32, 2^-23 of the partial sum each."""
    x, w = codes(depth, 300, 1, 0.05), codes(depth, 260, 2, 0.002)
    dy = (1e-3 * torch.randn(depth, 264, device="cuda", generator=gen(5))).to(BF)
    dw = q8.linear_dw(handle, dy, x, dtype=F32).double()
    want = dy.double().T @ dec(x)
    assert float((dw - want).norm() / want.norm()) <= 16 * 2.0 ** -23
    dyt = (1e-3 * torch.randn(200, depth, device="cuda", generator=gen(6))).to(BF)
    dx = q8.linear_dx(handle, dyt, w, dtype=F32).double()
    want = dyt.double() @ dec(w)
    assert float((dx - want).norm() / want.norm()) <= 16 * 2.0 ** -23


@pytest.mark.parametrize("t", [1, 5, 130])
def test_linear_longest_sum_of_largest_codes(handle, t):
    """127^2 * 131072 fits 32 bits: no sum wraps or saturates."""
    k, n = 131072, 40
    x, w = codes(t, k, 1), codes(n, k, 2)
    x.q.fill_(127), w.q.fill_(-127)
    x.scale.fill_(1.0), w.scale.fill_(1.0)
    out = q8.linear(handle, x, w, dtype=F32)
    assert (out.double() == float(np.float32(-127 * 127 * k))).all()


def test_products_carry_what_is_not_finite(handle):
    x, w = codes(40, 64, 1), codes(50, 64, 2)
    x.scale[7] = float("nan")
    x.q[7] = 0
    out = q8.linear(handle, x, w, dtype=F32)
    assert torch.isnan(out[7]).all() and int(torch.isnan(out).sum()) == 50
    dy = torch.ones(40, 50, device="cuda", dtype=BF)
    dy[3, 4] = float("nan")
    dx = q8.linear_dx(handle, dy, w, dtype=F32)
    assert torch.isnan(dx[3]).all() and int(torch.isnan(dx).sum()) == 64
    dw = q8.linear_dw(handle, dy, codes(40, 64, 1), dtype=F32)
    assert torch.isnan(dw[4]).all() and int(torch.isnan(dw).sum()) == 64


# ---- lengths of zero, streams, capture -------------------------------------------------------------------------------
def test_no_rows(handle):
    x = torch.empty(0, 48, device="cuda")
    w = torch.ones(48, device="cuda")
    o = q8.norm(handle, x, w, residual=x, values=True)
    assert o.rows.q.shape == (0, 48) and o.values.shape == (0, 48)
    dx, dw = q8.norm_backward(handle, x, x, w, o.rstd)
    assert dx.shape == (0, 48) and (dw == 0).all()
    a = q8.act(handle, x, "silu_gated", checkpoint=True)
    assert q8.act_backward(handle, torch.empty(0, 24, device="cuda"), a.checkpoint).shape == (0, 48)
    r, wt = q8.quantize_rows(handle, x), codes(32, 48, 1)
    assert q8.linear(handle, r, wt).shape == (0, 32)
    dy = torch.empty(0, 32, device="cuda", dtype=BF)
    assert q8.linear_dx(handle, dy, wt).shape == (0, 48)
    assert (q8.linear_dw(handle, dy, r) == 0).all() and (q8.bias_grad(handle, dy) == 0).all()


def test_another_stream_and_a_captured_graph(handle):
    x, res, w = hidden(64, 512, 1, BF), hidden(64, 512, 2, BF), torch.ones(512, device="cuda")
    wt, dy = codes(256, 512, 3), torch.randn(64, 256, device="cuda", generator=gen(4)).to(BF)
    side = torch.cuda.Stream()
    own = stq.Handle()

    def work(**kw):
        n = q8.norm(own, x, w, residual=res, **kw)
        y = q8.linear(own, n.rows, wt, **kw)
        return n.h, y, q8.linear_dx(own, dy, wt, **kw), q8.linear_dw(own, dy, n.rows, **kw), q8.bias_grad(own, dy, **kw)

    want = work()
    torch.cuda.synchronize()
    got = work(stream=side)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = work()
    x.copy_(hidden(64, 512, 9, BF))
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(work(), cap):
        assert torch.equal(a, b)
    own.device_status()
    own.close()


def test_offsets_beyond_32_bits(handle):
    """Rows 2^31 elements apart: the third begins 2^32 elements into its buffer."""
    ld = 2 ** 31 + 8
    big = torch.zeros(2 * ld + 512, dtype=BF, device="cuda")
    x = hidden(3, 512, 1, BF)
    far = big.as_strided((3, 512), (ld, 1))
    far.copy_(x)
    w, wt = torch.ones(512, device="cuda"), codes(512, 64, 2)
    for a, b in ((q8.norm(handle, far, w, values=True), q8.norm(handle, x, w, values=True)),):
        assert torch.equal(a.rows.q, b.rows.q) and torch.equal(a.values, b.values)
    a, b = q8.act(handle, far, "silu_gated", checkpoint=True), q8.act(handle, x, "silu_gated", checkpoint=True)
    assert torch.equal(a.rows.q, b.rows.q) and torch.equal(a.checkpoint.q[:, :, :256], b.checkpoint.q[:, :, :256])
    assert torch.equal(q8.quantize_rows(handle, far).q, q8.quantize_rows(handle, x).q)
    assert torch.equal(q8.linear_dx(handle, far, wt), q8.linear_dx(handle, x, wt))
    assert torch.equal(q8.linear_dw(handle, far, codes(3, 64, 3)), q8.linear_dw(handle, x, codes(3, 64, 3)))
    assert torch.equal(q8.bias_grad(handle, far), q8.bias_grad(handle, x))
    rstd = torch.ones(3, device="cuda")
    a, b = q8.norm_backward(handle, far, far, w, rstd), q8.norm_backward(handle, x, x, w, rstd)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("t,n,k", [(1, 70, 41), (7, 70, 41), (40, 77, 131), (300, 1283, 769), (2500, 1285, 1030), (8200, 1603, 1603)])
def test_what_lies_between_rows_does_not_matter(handle, t, n, k):
    """Codes and gradients whose rows are followed by anything up to their pitch: the largest codes, NaN."""
    def dirty(r):
        rows, cols = r.q.shape
        full = torch.full((rows, (cols + 15) // 16 * 16), 127, dtype=torch.int8, device="cuda")
        full[:, :cols] = r.q
        return q8.Rows8(full[:, :cols], r.scale)

    def clean(r):
        rows, cols = r.q.shape
        full = torch.zeros((rows, (cols + 15) // 16 * 16), dtype=torch.int8, device="cuda")
        full[:, :cols] = r.q
        return q8.Rows8(full[:, :cols], r.scale)

    x, w = codes(t, k, 1, 0.05), codes(n, k, 2, 0.002)
    dy = torch.randn(t, n, device="cuda", generator=gen(3)).to(BF)
    wide = torch.full((t, (n + 7) // 8 * 8), float("nan"), device="cuda", dtype=BF)
    wide[:, :n] = dy
    for dtype in (F32, BF):
        assert torch.equal(q8.linear(handle, dirty(x), dirty(w), dtype=dtype), q8.linear(handle, clean(x), clean(w), dtype=dtype))
        for g in (dy, wide[:, :n]):
            dx, dw = q8.linear_dx(handle, g, dirty(w), dtype=dtype), q8.linear_dw(handle, g, dirty(x), dtype=dtype)
            assert torch.equal(dx, q8.linear_dx(handle, dy, clean(w), dtype=dtype))
            assert torch.equal(dw, q8.linear_dw(handle, dy, clean(x), dtype=dtype))
    assert torch.equal(q8.bias_grad(handle, wide[:, :n]).isnan(), torch.zeros(n, dtype=torch.bool, device="cuda"))


@pytest.mark.parametrize("extra", [8, 3, 1])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("t,n,k", [(5, 72, 40), (90, 136, 264), (700, 1030, 520), (700, 1032, 513)])
def test_results_with_a_pitch_leave_what_lies_between_rows(handle, t, n, k, dtype, extra):
    """The C calls write rows of any pitch, on any aligned address, and nothing between them."""
    L, h, dt = q8._lib(), handle._h, 0 if dtype == F32 else 1
    x, w = codes(t, k, 1, 0.05), codes(n, k, 2, 0.002)
    dy = torch.randn(t, n, device="cuda", generator=gen(3)).to(BF)

    def into(rows, cols, call):
        ld = cols + extra
        buf = torch.full((rows * ld + 64,), 7.0, device="cuda").to(dtype)
        for shift in (0, 1, 8):
            buf.fill_(7.0)
            assert call(buf.data_ptr() + shift * buf.element_size(), ld) == 0
            body = buf[shift:shift + rows * ld].view(rows, ld)
            assert (body[:, cols:] == 7.0).all() and (buf[:shift] == 7.0).all() and (buf[shift + rows * ld:] == 7.0).all()
            yield body[:, :cols]

    P = torch.Tensor.data_ptr
    ldx, ldw = x.q.stride(0), w.q.stride(0)
    for got in into(t, n, lambda o, ld: L.stq_q8_linear(h, P(x.q), ldx, P(x.scale), P(w.q), ldw, P(w.scale), None, t, n, k, o, ld, dt, None)):
        assert torch.equal(got, q8.linear(handle, x, w, dtype=dtype))
    for got in into(t, k, lambda o, ld: L.stq_q8_linear_dx(h, P(dy), n, P(w.q), ldw, P(w.scale), t, n, k, o, ld, dt, None)):
        assert torch.equal(got, q8.linear_dx(handle, dy, w, dtype=dtype))
    for got in into(n, k, lambda o, ld: L.stq_q8_linear_dw(h, P(dy), n, P(x.q), ldx, P(x.scale), t, n, k, o, ld, dt, None)):
        assert torch.equal(got, q8.linear_dw(handle, dy, x, dtype=dtype))
    z = hidden(t, 2 * k, 4, dtype)
    ck = q8.act(handle, z, "silu_gated", checkpoint=True).checkpoint
    da = hidden(t, k, 5, dtype)
    for got in into(t, 2 * k, lambda o, ld: L.stq_q8_act_backward(h, P(da), k, 1, dt, t, k, P(ck.q), ck.q.shape[2], P(ck.scale), o, ld, None)):
        assert torch.equal(got, q8.act_backward(handle, da, ck))
    g, rstd, dw = torch.ones(k, device="cuda"), torch.ones(t, device="cuda"), torch.empty(k, device="cuda")
    hh = hidden(t, k, 6, dtype)
    for got in into(t, k, lambda o, ld: L.stq_q8_norm_backward(h, P(da), k, P(hh), k, P(g), P(rstd), None, 0, dt, t, k, o, ld, P(dw), None)):
        xh, up = hh.double(), da.double()          # (rstd and weight are 1)
        want, size = up - xh * (up * xh).mean(1, keepdim=True), up.abs() + xh.abs() * (up * xh).abs().mean(1, keepdim=True)
        assert ((got.double() - want).abs() <= 64 * U * size + (UB * 1.01 * want.abs() if dtype == BF else 0)).all()


# ---- refusals --------------------------------------------------------------------------------------------------------
def test_refusals_of_the_binding(handle):
    x, w = hidden(4, 64, 1), torch.ones(64, device="cuda")
    ok8 = codes(4, 64, 1)
    bad = [
        (lambda: q8.norm(handle, x.half(), w), "float32 or bfloat16"),
        (lambda: q8.norm(handle, x, w.to(BF)), "weight"),
        (lambda: q8.norm(handle, x, w[:32]), "weight"),
        (lambda: q8.norm(handle, x, w, residual=x[:3]), "4 rows"),
        (lambda: q8.norm(handle, x, w, residual=x.to(BF)), "residual"),
        (lambda: q8.norm(handle, x.t(), torch.ones(4, device="cuda")), "unit stride"),
        (lambda: q8.norm(handle, x[0], w), "matrix"),
        (lambda: q8.norm(handle, x.cpu(), w), "device"),
        (lambda: q8.quantize_rows(handle, x[:1].expand(4, 64)), "overlap"),
        (lambda: q8.act(handle, x, "relu"), "kind"),
        (lambda: q8.act(handle, x[:, :63], "silu_gated"), "even"),
        (lambda: q8.linear(handle, ok8, codes(4, 48, 1)), "64 columns"),
        (lambda: q8.linear(handle, ok8, ok8, dtype=torch.float16), "float32 or bfloat16"),
        (lambda: q8.linear(handle, q8.Rows8(x, ok8.scale), ok8), "int8"),
        (lambda: q8.linear(handle, q8.Rows8(ok8.q, ok8.scale[:3]), ok8), "scale"),
        (lambda: q8.linear_dx(handle, x, codes(64, 32, 1)), "bfloat16"),
        (lambda: q8.linear_dw(handle, x[:3].to(BF), ok8), "4 rows"),
    ]
    before = handle.launch_count
    for call, what in bad:
        with pytest.raises(ValueError, match=what):
            call()
    a = q8.act(handle, x, "gelu", checkpoint=True).checkpoint
    with pytest.raises(ValueError, match="parts"):
        q8.act_backward(handle, x[:, :64], a._replace(kind="silu_gated"))
    assert handle.launch_count == before + 1      # (the one valid call above)


def test_refusals_of_the_library(handle):
    L, h = q8._lib(), handle._h
    x, w, big = torch.zeros(8, 64, device="cuda"), torch.ones(64, device="cuda"), torch.zeros(1 << 16, device="cuda")
    q = torch.zeros(8, 64, dtype=torch.int8, device="cuda")
    s, f = torch.zeros(64, device="cuda"), big.data_ptr()
    X, W, Q, S = x.data_ptr(), w.data_ptr(), q.data_ptr(), s.data_ptr()
    NULL, ALIGN, ALIAS, NUMEL, ARG, LARGE = -1, -4, -5, -6, -9, -12

    def rows(h=h, x=X, ldx=64, dt=0, r=8, c=64, q=Q, ldq=64, s=S):
        return L.stq_q8_rows(h, x, ldx, dt, r, c, q, ldq, s, None)

    before = handle.launch_count
    assert rows(h=None) == NULL and rows(x=None) == NULL and rows(q=None) == NULL and rows(s=None) == NULL
    assert rows(dt=2) == ARG and rows(ldx=63) == ARG and rows(ldq=48) == ARG and rows(c=0) == NUMEL
    assert rows(q=Q + 8) == ALIGN and rows(ldq=72) == ALIGN and rows(x=X + 1) == ALIGN and rows(s=S + 2) == ALIGN
    assert rows(r=1 << 31) == LARGE and rows(c=(1 << 24) + 16, ldx=1 << 25, ldq=1 << 25) == LARGE
    assert rows(q=X) == ALIAS and rows(s=X + 4) == ALIAS

    def norm(eps=1e-6, res=None, hs=None, w=W, rstd=f, v=None, ldv=64):
        return L.stq_q8_norm(h, X, 64, res, 64, w, eps, 0, 8, 64, hs, 64, rstd, Q, 64, S, v, ldv, None)

    assert norm(eps=0.0) == ARG and norm(eps=float("nan")) == ARG and norm(w=None) == NULL and norm(rstd=None) == NULL
    assert norm(res=f) == NULL and norm(hs=f) == NULL and norm(res=f + 4096, hs=X) == ALIAS and norm(v=f + 4096, ldv=8) == ARG
    nb = lambda c=64, dw=S, dx=f: L.stq_q8_norm_backward(h, X, 64, X, 64, W, W, None, 0, 0, 8, c, dx, 64, dw, None)  # noqa: E731
    assert nb(dw=None) == NULL and nb(dx=X) == ALIAS and nb(c=49153) == LARGE
    ac = lambda kind=2, ck=None, cs=None: L.stq_q8_act(h, X, 64, kind, 0, 8, 64, Q, 64, S, None, 0, ck, 64, cs, None)  # noqa: E731
    assert ac(kind=0) == ARG and ac(kind=1) == ARG and ac(ck=f) == NULL and ac(ck=Q, cs=f) == ALIAS
    li = lambda k=64, out=f, dt=0, n=8: L.stq_q8_linear(h, Q, 64, S, Q, 64, S, None, 8, n, k, out, 64, dt, None)  # noqa: E731
    assert li(k=0) == NUMEL and li(n=0) == NUMEL and li(out=None) == NULL and li(dt=2) == ARG and li(out=Q) == ALIAS
    assert L.stq_q8_linear(h, Q, 1 << 18, S, Q, 1 << 18, S, None, 1, 1, 131073, f, 64, 0, None) == LARGE
    assert L.stq_q8_linear_dx(h, X + 1, 64, Q, 64, S, 8, 8, 64, f, 64, 0, None) == ALIGN
    assert L.stq_q8_linear_dw(h, X, 64, Q, 64, S, 8, 8, 64, X, 64, 0, None) == ALIAS
    assert L.stq_q8_bias_grad(h, X, 64, 0, 8, 64, None, None) == NULL
    assert handle.launch_count == before
    with pytest.raises(stq.StqError) as e:
        q8.norm(handle, x, w, eps=-1.0)
    assert e.value.code == ARG
