"""The 8-bit operators at the edges of the numbers' range, and after calls that failed."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2604_06836_b200 import q8, stq   # noqa: E402

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24          # half an ulp of fp32


@pytest.fixture(scope="module")
def handle():
    h = stq.Handle()
    yield h
    h.device_status()
    h.close()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def backward(h, t, n, k, seed):
    """One of each backward call that uses the workspace, as a function of nothing, and the inputs it reads."""
    g = gen(seed)
    dy = torch.randn(t, n, device="cuda", generator=g).to(BF)
    x, w = (q8.quantize_rows(h, torch.randn(r, k, device="cuda", generator=g)) for r in (t, n))
    hid, weight = torch.randn(t, n, device="cuda", generator=g).to(BF), torch.ones(n, device="cuda")
    rstd = hid.float().square().mean(1).rsqrt()

    def call():
        return [q8.linear_dx(h, dy, w, dtype=F32), q8.linear_dw(h, dy, x, dtype=F32), q8.linear_dw(h, dy, x),
                q8.bias_grad(h, dy), *q8.norm_backward(h, dy, hid, weight, rstd)]
    return call, dy


# ---- workspace -------------------------------------------------------------------------------------------------------
def test_a_workspace_that_cannot_be_had_leaves_the_handle_usable():
    """The sizes ask for a copy of half a terabyte (dy lies on an odd address): refused before anything is launched."""
    h = stq.Handle()
    L, buf, q, s = q8._lib(), torch.zeros(4096, device="cuda"), torch.zeros(128, 64, dtype=torch.int8, device="cuda"), torch.ones(128, device="cuda")
    before = h.launch_count
    rc = L.stq_q8_linear_dx(h._h, buf.data_ptr() + 2, 128, q.data_ptr(), 64, s.data_ptr(), 2 ** 31 - 1, 128, 64,
                            1 << 46, 64, 1, None)      # (an address nothing lives at; it is compared and never touched)
    assert rc == -8 and h.launch_count == before
    x = torch.randn(5, 64, device="cuda", generator=gen(1))
    r = q8.quantize_rows(h, x)
    assert int(r.q.abs().max()) == 127
    h.device_status()
    h.close()


def test_a_captured_graph_outlives_the_growth_of_the_workspace():
    h = stq.Handle()
    small, dy = backward(h, 300, 261, 128, 1)                  # (odd rows of dy: copied to the workspace)
    small()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = small()
    grown = []
    for t, n, k in ((2000, 1285, 640), (5000, 1285, 2056)):    # more workspace twice over
        large, _ = backward(h, t, n, k, 2)
        grown.append((large, large()))
    # whatever had been freed would be handed out here
    other = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(64)]
    dy.copy_(torch.randn(dy.shape, device="cuda", generator=gen(3)).to(BF))
    graph.replay()
    torch.cuda.synchronize()
    assert all(bool((o == 3.0).all()) for o in other)
    own = stq.Handle()
    fresh, dy2 = backward(own, 300, 261, 128, 1)
    dy2.copy_(dy)
    for a, b in zip(captured, fresh()):
        assert torch.equal(a, b)
    for large, before in grown:
        for a, b in zip(large(), before):
            assert torch.equal(a, b)
    h.device_status(), own.device_status()
    del graph
    h.close(), own.close()


@pytest.mark.parametrize("mode", ["global", "thread_local", "relaxed"])
def test_the_workspace_grows_during_a_capture(mode):
    h, own = stq.Handle(), stq.Handle()
    first, _ = backward(h, 130, 261, 128, 4)
    first()                                                    # (a buffer that the capture replaces)
    call, dy = backward(h, 300, 261, 128, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode=mode):
        got = call()
    large, _ = backward(h, 2000, 1285, 640, 2)
    large()
    fresh, dy2 = backward(own, 300, 261, 128, 1)
    for seed in (5, 6):
        dy.copy_(torch.randn(dy.shape, device="cuda", generator=gen(seed)).to(BF))
        dy2.copy_(dy)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, fresh()):
            assert torch.equal(a, b)
    h.device_status(), own.device_status()
    del graph
    h.close(), own.close()


# ---- norm ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,cols", [(4, 96), (3, 257), (2, 2048), (1100, 1536), (2, 16640)])
@pytest.mark.parametrize("size,eps", [(1e-32, 1e-6), (1e-33, 1e-12), (3e-30, 1e-6), (1e-35, 1e-6)])
def test_norm_of_small_rows(handle, rows, cols, dtype, size, eps):
    """eps lifts small rows: whether a row is stored as zeros goes by the norm's result, not by h * weight."""
    x = (size * torch.randn(rows, cols, device="cuda", generator=gen(cols))).to(dtype)
    w = 1 + 0.1 * torch.randn(cols, device="cuda", generator=gen(2))
    out = q8.norm(handle, x, w, eps=eps, values=True)
    xd = x.double()
    y = xd * (xd.square().mean(1, keepdim=True) + eps).rsqrt() * w.double()
    top = y.abs().amax(1)
    clear = (top / 2.0 ** -100 - 1).abs() > 1e-5          # (a row on the limit may go either way)
    zero = top < 2.0 ** -100
    scale, codes = out.rows.scale.double(), out.rows.q.double()
    assert (scale[zero & clear] == 0).all() and (codes[zero & clear] == 0).all()
    keep = ~zero & clear
    # rstd, the product with it, the scale: a few roundings each; codes off by that much next to a tie
    assert ((scale - top / 127).abs()[keep] <= 16 * U * top[keep] / 127).all()
    quot = y[keep] * (127 / top[keep])[:, None]
    assert ((codes[keep] - quot).abs() <= 0.5 + 127 * 16 * U).all()
    assert torch.equal(out.values, (out.rows.q.float() * out.rows.scale[:, None]).to(BF))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,cols", [(4736, 200), (4737, 200), (2368, 512), (2369, 512), (2369, 510), (676, 1600), (677, 1600), (677, 1601),
                                       (296, 4096), (297, 4096), (148, 8192), (149, 8192), (300, 8190), (5, 8200), (300, 10240), (300, 16384),
                                       (5, 16392), (300, 16392)])
def test_row_kernels_where_their_shape_changes(handle, rows, cols, dtype):
    """The same rows alone and among others, on both sides of every limit: the norm, the gated activation with its
    checkpoint, plain rows."""
    g = gen(rows + cols)
    x, res = (torch.randn(rows, cols, device="cuda", generator=g).to(dtype) for _ in range(2))
    w = 1 + 0.1 * torch.randn(cols, device="cuda", generator=g)
    out = q8.norm(handle, x, w, residual=res, eps=1e-6)
    hd = x.double() + res.double()
    rstd = (hd.square().mean(1) + 1e-6).rsqrt()
    y = hd * rstd[:, None] * w.double()
    top = y.abs().amax(1, keepdim=True)
    assert torch.equal(out.h, (x.float() + res.float()).to(dtype)) and ((out.rstd.double() - rstd).abs() <= 40 * U * rstd).all()
    assert ((out.rows.scale.double() - top[:, 0] / 127).abs() <= 48 * U * top[:, 0] / 127).all()
    assert ((out.rows.q.double() - y * (127 / top)).abs() <= 0.5 + 127 * 5 * U).all()
    few = slice(rows - 2, rows)
    r = q8.quantize_rows(handle, x)
    z = torch.cat([x, res], dim=1)
    a = q8.act(handle, z, "silu_gated", checkpoint=True)
    r2, a2 = q8.quantize_rows(handle, x[few]), q8.act(handle, z[few], "silu_gated", checkpoint=True)
    assert torch.equal(r.q[few], r2.q) and torch.equal(r.scale[few], r2.scale)
    assert torch.equal(a.rows.q[few], a2.rows.q) and torch.equal(a.rows.scale[few], a2.rows.scale)
    assert torch.equal(a.checkpoint.q[few, :, :cols], a2.checkpoint.q[:, :, :cols]) and torch.equal(a.checkpoint.scale[few], a2.checkpoint.scale)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("cols", [4096, 4097, 4098, 4104, 5121, 8190, 8191, 8192, 8193, 8194, 8200])
@pytest.mark.parametrize("rows", [3, 300])
def test_norm_backward_where_its_variants_change(handle, rows, cols, dtype):
    g = gen(rows + cols)
    h, dy, dres = ((s * torch.randn(rows, cols, device="cuda", generator=g)).to(dtype) for s in (2.0, 1e-3, 1e-3))
    w = 1 + 0.1 * torch.randn(cols, device="cuda", generator=g)
    rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
    dx, dw = q8.norm_backward(handle, dy, h, w, rstd, dres=dres)
    rs = rstd.double()[:, None]
    xh, up = h.double() * rs, dy.double() * w.double()
    want = rs * (up - xh * (up * xh).mean(1, keepdim=True)) + dres.double()
    # a sum of `cols` terms in a tree of at most 8 * 32 and log2 steps; the mean of terms of either sign is small beside them
    size = rs * (up.abs() + xh.abs() * (up * xh).abs().mean(1, keepdim=True)) + dres.double().abs()
    tol = 64 * U * size + (2.0 ** -8 * 1.01 * want.abs() if dtype == BF else 0)
    assert ((dx.double() - want).abs() <= tol).all()
    assert ((dw.double() - (dy.double() * xh).sum(0)).abs() <= 64 * U * (dy.double() * xh).abs().sum(0)).all()
    again = q8.norm_backward(handle, dy, h, w, rstd, dres=dres)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


# ---- products --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("t", [1, 3, 12, 130, 300, 3000])
def test_scales_whose_product_leaves_the_range(handle, t):
    """The result is in range although the product of its two scales is not: neither lost digits nor NaN."""
    n, k = 264, 320
    g = gen(t)
    codes = [q8.alloc_rows(r, k, "cuda") for r in (t, n)]
    for r in codes:
        r.q.copy_(torch.randint(-127, 128, r.q.shape, device="cuda", generator=g, dtype=torch.int32).to(torch.int8))
    x, w = codes
    w.q[5] = 0                                             # a sum of zero
    for sx, sw in ((2.0 ** -90 * 1.1, 2.0 ** -50 * 1.3), (2.0 ** 60 * 1.1, 2.0 ** 50 * 1.3), (2.0 ** 80 * 1.1, 2.0 ** 60 * 1.3)):
        x.scale.fill_(sx), w.scale.fill_(sw)
        sums = x.q.double() @ w.q.double().T
        want = sums * x.scale.double()[:, None] * w.scale.double()
        got = q8.linear(handle, x, w, dtype=F32).double()
        fits = (want.abs() < 3.3e38) & ((want.abs() > 2.0 ** -120) | (sums == 0))
        assert fits.any()
        assert ((got - want).abs()[fits] <= 4 * U * want.abs()[fits]).all()
        assert (got[:, 5] == 0).all()


# ---- activations -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("kind", ["silu_gated", "gelu"])
@pytest.mark.parametrize("cols", [128, 131, 258])
def test_act_backward_of_large_inputs(handle, kind, dtype, cols):
    """The derivative of a saturated activation is 0 or 1, up to the type's largest and lowest values."""
    parts = 2 if kind == "silu_gated" else 1
    sizes = [15.0, 40.0, 1e6, 2e13, 1e15, 1e20, 3.3e38]
    z = torch.randn(2 * len(sizes), parts * cols, device="cuda", generator=gen(5))
    for i, s in enumerate(sizes):
        z[2 * i, 3], z[2 * i + 1, 3] = s, -s
    ck = q8.act(handle, z.to(dtype), kind, checkpoint=True).checkpoint
    da = torch.randn(z.shape[0], cols, device="cuda", generator=gen(6)).to(dtype)
    dz = q8.act_backward(handle, da, ck).double()
    kept = ck.values().double().requires_grad_(True)
    if kind == "silu_gated":
        a = kept[:, :cols] * torch.sigmoid(kept[:, :cols]) * kept[:, cols:]
    else:
        a = torch.nn.functional.gelu(kept, approximate="tanh")
    a.backward(da.double())
    want = kept.grad
    assert torch.isfinite(dz).all()
    ok = want.abs() < 3.3e38
    kd = kept.detach().abs()
    # where the sigmoid is not saturated the size of the terms, |g| <= 40, carries the exponent's rounding
    size = da.double().abs().repeat(1, parts) * (1 + kd.clamp(max=40)) * (1 + (kd[:, cols:].repeat(1, 2) if parts == 2 else 0))
    tol = 1e-5 * size + 1e-5 * want.abs() + (2.0 ** -8 * 1.01 * want.abs() if dtype == BF else 0)
    assert ((dz - want).abs() <= tol)[ok].all()
