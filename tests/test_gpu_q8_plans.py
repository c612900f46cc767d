"""Gradients of the 8-bit product in every form that their plan can take, against 64 bits, in the 2-norm.

A bound on single elements relative to the sum of the terms' magnitudes is loose: it hides a term that was left out.  The
2-norm shows one term of a thousand as 3 % of the result.  A rounding to bf16 is at most 2^-8 / sqrt(3) in the mean square
(numbers at the low end of their binade, errors evenly spread); the operand's and the result's are independent.  An fp32
result is held to 16 steps of the matrix unit at full size, 2^-23 each.  Single rows and columns (of 100 elements and
more) are held to twice that, since their own size scatters.

The shapes are chosen so that on 148 SMs the plan has whole tiles ("full" of them), tiles whose sums are shared and joined,
or both, in CTA pairs or not, with the 8-bit operand converted inside the product or ahead of it."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2604_06836_b200 import q8, stq   # noqa: E402

BF, F32 = torch.bfloat16, torch.float32
NORM = {BF: (2 ** 0.5) * 2.0 ** -8 / 3 ** 0.5, F32: 16 * 2.0 ** -23}


@pytest.fixture(scope="module")
def handle():
    h = stq.Handle()
    if h.sm_count != 148:
        pytest.skip("the plans are those of 148 SMs")
    yield h
    h.device_status()
    h.close()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def codes(rows, cols, seed, scale):
    g = gen(seed)
    r = q8.alloc_rows(rows, cols, "cuda")
    r.q.copy_(torch.randint(-127, 128, (rows, cols), device="cuda", generator=g, dtype=torch.int32).to(torch.int8))
    r.scale.copy_(scale * (0.5 + torch.rand(rows, device="cuda", generator=g)))
    return r


def check(got, want, dtype):
    off = got.double() - want
    tol = NORM[dtype]
    assert float(off.norm() / want.norm()) <= tol
    for dim in (d for d in (0, 1) if want.shape[d] >= 100):
        assert bool((off.norm(dim=dim) <= 2 * tol * want.norm(dim=dim)).all())


# t, n, k; result; whole tiles or not, pairs or not, conversion ahead or not
DX = [
    (8192, 6400, 1600, BF, "full shared pairs ahead"),
    (8191, 6401, 1603, BF, "full shared pairs ahead"),
    (6336, 4856, 209, BF, "shared pairs ahead"),
    (6208, 2190, 517, BF, "full shared pairs ahead"),
    (3168, 4721, 138, BF, "shared pairs"),
    (3776, 707, 1280, BF, "full shared pairs"),
    (3775, 712, 1277, BF, "full shared pairs"),
    (143, 3008, 1641, BF, "shared"),
    (513, 4480, 3743, BF, "full shared"),
    (128, 1216, 128, BF, "shared"),
    (296, 3520, 3156, BF, "full shared"),
    (300, 1283, 769, BF, "full"),
    (8192, 6400, 1600, F32, "full shared pairs"),
    (8191, 6401, 1603, F32, "full shared pairs"),
    (704, 705, 3200, F32, "full shared pairs"),
    (138, 2511, 1664, F32, "shared pairs"),
    (130, 2916, 4800, F32, "full shared"),
    (111, 810, 128, F32, "shared"),
]
DW = [
    (8192, 6400, 1600, BF, "full shared pairs ahead"),
    (8191, 6401, 1603, BF, "full shared pairs ahead"),
    (5376, 6208, 199, BF, "shared pairs ahead"),
    (2356, 6272, 542, BF, "full shared pairs ahead"),
    (6272, 139, 2496, BF, "shared pairs"),
    (731, 910, 4800, BF, "full shared pairs"),
    (731, 912, 4799, BF, "full shared pairs"),
    (3848, 143, 1600, BF, "shared"),
    (4386, 275, 6336, BF, "full shared"),
    (1306, 111, 136, BF, "shared"),
    (4224, 262, 3200, BF, "full shared"),
    (300, 1283, 769, BF, "full"),
    (8192, 6400, 1600, F32, "full shared pairs"),
    (8191, 6401, 1603, F32, "full shared pairs"),
    (768, 448, 4810, F32, "full shared pairs"),
    (2224, 152, 1623, F32, "shared pairs"),
    (2752, 155, 4780, F32, "full shared"),
    (942, 128, 128, F32, "shared"),
]


def gradient(handle, call, dy, r, dtype, form, want):
    before = handle.launch_count
    got = call(handle, dy, r, dtype=dtype)
    # a copy of dy with rows that are not whole pieces of 16 bytes, the conversion, the product, the joining
    assert handle.launch_count - before == (dy.shape[1] % 8 != 0) + ("ahead" in form) + 1 + ("shared" in form)
    check(got, want, dtype)
    assert torch.equal(got, call(handle, dy, r, dtype=dtype))


@pytest.mark.parametrize("t,n,k,dtype,form", DX)
def test_input_gradient(handle, t, n, k, dtype, form):
    w = codes(n, k, n, 0.002)
    dy = (1e-3 * torch.randn(t, n, device="cuda", generator=gen(t))).to(BF)
    gradient(handle, q8.linear_dx, dy, w, dtype, form, (dy.double() * w.scale.double()) @ w.q.double())


@pytest.mark.parametrize("t,n,k,dtype,form", DW)
def test_weight_gradient(handle, t, n, k, dtype, form):
    x = codes(t, k, k, 0.05)
    dy = (1e-3 * torch.randn(t, n, device="cuda", generator=gen(t))).to(BF)
    gradient(handle, q8.linear_dw, dy, x, dtype, form, (dy.double() * x.scale.double()[:, None]).T @ x.q.double())


@pytest.mark.parametrize("t,n,k", [(1003, 1283, 769), (513, 1000, 264), (130, 2304, 768), (17, 130, 769), (2500, 1285, 1030)])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_no_token_and_no_channel_is_left_out(handle, t, n, k, dtype):
    """The last tokens and channels weigh as much as all others together: without one the result is half as large."""
    x, w = codes(t, k, 1, 0.05), codes(n, k, 2, 0.002)
    for at in (0, -1, -2, -3):
        dy = torch.randn(t, n, device="cuda", generator=gen(5))
        dy[at] *= t ** 0.5
        check(q8.linear_dw(handle, dy.to(BF), x, dtype=dtype), (dy.to(BF).double() * x.scale.double()[:, None]).T @ x.q.double(), dtype)
        dy = torch.randn(t, n, device="cuda", generator=gen(6))
        dy[:, at] *= n ** 0.5
        check(q8.linear_dx(handle, dy.to(BF), w, dtype=dtype), (dy.to(BF).double() * w.scale.double()) @ w.q.double(), dtype)
