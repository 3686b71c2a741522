"""Products of values held in 8-bit floating point against the same values' products in 64 bits.

Tolerances.  Each product of two values and their scales is exact in 32 bits.  To a float32 output
the values go as bfloat16, whose instructions add 32 of them in 32 bits: at most 128 roundings
of 2^-24 of what is added for each block of k, and one rounding of the sum; splits of a sum add at most 16 more.
So a result is off by at most (128 + blocks + 16) 2^-24 times the sum of magnitudes, and half a step of
its type, eps / 2.  To a 16-bit output the 8-bit instruction adds eight products after bringing them to the
largest one's exponent, 2^E <= |largest| < 2^(E + 2), and cutting each off below 2^(E - 13); eight cuts lose less
than 8 * 2^(E - 13) = 2^(E - 10), at most 2^-10 of the eight's sum of magnitudes.  The groups' sums are added
in 32 bits, 16 for a block: (16 + blocks + 16) 2^-24 more."""

import pytest
import torch

from tests.scaled_form import hold, in_order, scaled, values

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
TINY = {torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25, torch.float32: 1e-37}
SHAPES = [(1, 1, 1), (1, 8192, 256), (1, 130, 5000), (3, 17, 129), (16, 64, 128), (17, 100, 300),
          (32, 33, 1000), (33, 64, 64), (40, 500, 2059), (64, 128, 128), (100, 7, 40), (129, 257, 385),
          (333, 501, 700), (300, 520, 4096), (1000, 48, 16), (700, 900, 130)]


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def make(rows, k, seed):
    """Rows and blocks of different sizes."""
    g = torch.Generator().manual_seed(seed)
    size = torch.exp2(torch.randint(-4, 5, (rows, -(-k // 128)), generator=g).float())
    return torch.randn(rows, k, generator=g) * size.repeat_interleave(128, 1)[:, :k]


def near(got, a, b, what=""):
    half = torch.finfo(got.dtype).eps / 2
    want, size = a @ b.t(), a.abs() @ b.abs().t()
    blocks = -(-a.shape[1] // 128)
    work = (128 + blocks + 16) * 2.0 ** -24
    if got.dtype != torch.float32:
        work = 2.0 ** -10 + (16 + blocks + 16) * 2.0 ** -24
    off = (got.double().cpu() - want).abs()
    lim = want.abs() * half + size * work * (1 + half) + TINY[got.dtype]
    bad = ~(off <= lim)
    assert not bad.any(), "%s %d values, worst %g of the bound" % (what, int(bad.sum()),
                                                                   float((off / lim).max()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product(kr, m, n, k, dtype):
    a, b = make(m, k, m + k), make(n, k, n + k) / k ** 0.5
    va, vb = values(*hold(a)), values(*hold(b))
    contiguous = kr.scaled_matmul(scaled(kr, a), scaled(kr, b), dtype)
    near(contiguous, va, vb)
    roomy = kr.scaled_matmul(kr.scaled_hold(a.cuda()).plain, kr.scaled_hold(b.cuda()).plain, dtype)
    assert torch.equal(contiguous, roomy)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 40, 1024), (20, 40, 1024), (200, 300, 2000), (600, 700, 1024)])
def test_whole_numbers_are_exact(kr, m, n, k, dtype):
    """Small whole numbers, scales of different powers: every sum fits 24 bits, the products of a block's
    eight neighbours (0 or 1 to 64 of one unit) the 13 bits that are kept of them, so nothing rounds
    but the result."""
    g = torch.Generator().manual_seed(k)
    a, b = (torch.randint(-8, 9, (r, k), generator=g).double() for r in (m, n))
    ea, eb = (torch.randint(0, 3, (r, -(-k // 128)), generator=g) for r in (m, n))
    got = kr.scaled_matmul(kr.Scaled(a.to(torch.float8_e4m3fn).cuda(), in_order(ea + 127).cuda()),
                           kr.Scaled(b.to(torch.float8_e4m3fn).cuda(), in_order(eb + 127).cuda()), dtype)
    assert torch.equal(got.cpu(), (values(a, ea + 127) @ values(b, eb + 127).t()).to(dtype))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n", [(5, 40), (40, 300), (300, 300)])
def test_every_value(kr, m, n, dtype):
    """All 256 bytes but the NaN, and all scales whose products 32 bits hold: one product at a time."""
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn)
    every = every[torch.isfinite(every.float())]
    k = 254 * 128  # a value in each block, ones against them
    a = torch.zeros(m, k, dtype=torch.float64)
    a[m // 2, ::128] = every.double()
    ea = torch.full((m, 254), 127)
    ea[m // 2] = torch.arange(254) % 100 + 70
    for block in (0, 1, 126, 127, 200, 253):
        b = torch.zeros(n, k, dtype=torch.float64)
        b[n // 2, block * 128] = 1
        got = kr.scaled_matmul(kr.Scaled(a.to(torch.float8_e4m3fn).cuda(), in_order(ea).cuda()),
                               kr.Scaled(b.to(torch.float8_e4m3fn).cuda(),
                                         in_order(torch.full((n, 254), 127)).cuda()), dtype)
        want = torch.zeros(m, n, dtype=torch.float64)
        want[m // 2, n // 2] = a[m // 2, block * 128] * 2.0 ** float(ea[m // 2, block] - 127)
        assert torch.equal(got.double().cpu(), want), block


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 20, 140, 600])
def test_no_numbers(kr, m, dtype):
    """A block that holds no number spoils its row or column alone."""
    a, b = make(m, 700, 1), make(300, 700, 2)
    good = kr.scaled_matmul(kr.scaled_hold(a.cuda()).plain, kr.scaled_hold(b.cuda()).plain, dtype)
    a[m // 2, 300], b[17, 699] = float("inf"), float("nan")
    got = kr.scaled_matmul(kr.scaled_hold(a.cuda()).plain, kr.scaled_hold(b.cuda()).plain, dtype)
    bad = torch.zeros(m, 300, dtype=torch.bool)
    bad[m // 2], bad[:, 17] = True, True
    assert torch.equal(got.isnan().cpu(), bad)
    assert torch.equal(got.cpu()[~bad], good.cpu()[~bad])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(3, 50, 259), (200, 300, 259), (600, 700, 1040)])
def test_strides(kr, m, n, k, dtype):
    """Rows apart, unaligned, crossed, in more dimensions, scales in a larger tensor: the same bits."""
    a, b = make(m, k, 5), make(n, k, 6)
    want = kr.scaled_matmul(scaled(kr, a), scaled(kr, b), dtype)
    near(want, values(*hold(a)), values(*hold(b)))

    def moved(h, start, more):
        rows = h.q.shape[0]
        store = torch.full((rows, k + more), 0x7F, dtype=torch.uint8, device="cuda")  # NaN around
        q = store[:, start:start + k]
        q.copy_(h.q.view(torch.uint8))
        scale = torch.full((h.scale.shape[0], h.scale.shape[1] + 12), 255, dtype=torch.uint8,
                           device="cuda")
        scale[:, 4:-8] = h.scale
        return kr.Scaled(q.view(torch.float8_e4m3fn), scale[:, 4:-8])

    for start, more in ((0, 13), (1, 1), (16, 32 + -k % 16), (5, 100)):
        got = kr.scaled_matmul(moved(scaled(kr, a), start, more), moved(scaled(kr, b), start, more),
                               dtype)
        assert torch.equal(got, want), (start, more)
    ha = scaled(kr, a)
    crossed = kr.Scaled(ha.q.view(torch.uint8).t().contiguous().t().view(torch.float8_e4m3fn), ha.scale)
    assert torch.equal(kr.scaled_matmul(crossed, scaled(kr, b), dtype), want)
    if m == 600:
        x = kr.scaled_hold(a.reshape(20, 30, k).cuda()).plain
        got = kr.scaled_matmul(x, scaled(kr, b), dtype)
        assert got.shape == (20, 30, n) and torch.equal(got.reshape(m, n), want)


def test_gaps_between_output_rows(kr):
    """The C call to rows apart: their gaps and the rows behind stay."""
    import ctypes

    for m, n in ((5, 37), (150, 300)):
        a, b = scaled(kr, make(m, 300, 5)), scaled(kr, make(n, 300, 6))
        want = kr.scaled_matmul(a, b, torch.float32)
        out = torch.full((m + 1, n + 5), 7.0, device="cuda")
        ka, kb = kr._held(a, "a", 0)[0], kr._held(b, "b", 0)[0]
        p = kr.KrScaledProduct(m, n, 300, ka, kb)
        wsb = kr._lib.kr_scaled_matmul_workspace(p)
        ws, at = kr._scratch(wsb)
        assert kr._lib.kr_scaled_matmul(ctypes.byref(p), 0, out.data_ptr(), n + 5, at, wsb,
                                        kr._raw_stream(0)) == kr.KR_OK
        assert torch.equal(out[:m, :n], want)
        assert (out[m] == 7).all() and (out[:, n:] == 7).all()


def test_empty(kr):
    b = scaled(kr, make(40, 300, 6))
    a = kr.scaled_hold(torch.zeros(0, 300).cuda()).plain
    assert kr.scaled_matmul(a, b).shape == (0, 40)


def reference(x, w, dout):
    """Output and gradients in 64 bits, with what is summed and its size."""
    y = (values(*hold(x)), values(*hold(w, True)))
    dx = (values(*hold(dout)), values(*hold(w.t(), True)))
    dw = (values(*hold(dout.t())), values(*hold(x.t())))
    return y, dx, dw


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,hidden", [(1, 64, 40), (7, 129, 200), (40, 72, 56), (300, 257, 129),
                                               (260, 512, 384)])
def test_linear(kr, rows, width, hidden, dtype):
    x, dout = make(rows, width, 1).to(dtype), make(rows, hidden, 3).to(dtype)
    w = (make(hidden, width, 2) / width ** 0.5).to(dtype)
    y, dx, dw = reference(x, w, dout)
    xg, wg = x.cuda().requires_grad_(), w.cuda().requires_grad_()
    out = kr.scaled_linear(xg, wg)
    assert out.dtype == dtype
    near(out.detach(), *y, "y")
    out.backward(dout.cuda())
    near(xg.grad, *dx, "dx")
    near(wg.grad, *dw, "dw")
    one, two = kr.scaled_linear_backward(dout.cuda(), x.cuda(), w.cuda())
    assert torch.equal(one, xg.grad) and torch.equal(two, wg.grad)
    held = kr.scaled_hold(w.cuda(), square=True).plain
    with torch.no_grad():
        assert torch.equal(kr.scaled_linear(x.cuda(), held), out)
    xg.grad = wg.grad = None
    kr.scaled_linear(xg, w.cuda()).backward(dout.cuda())
    kr.scaled_linear(x.cuda(), wg).backward(dout.cuda())
    assert torch.equal(xg.grad, one) and torch.equal(wg.grad, two)


def test_linear_gradient_against_differences(kr):
    """Where holding leaves values as they are (small whole numbers, 448 in every block), the gradient is
    that of x w^T: against differences of the product in 64 bits, exact for a bilinear form."""
    g = torch.Generator().manual_seed(3)
    x, w, d = (torch.randint(-3, 4, s, generator=g).double() for s in ((5, 130), (9, 130), (5, 9)))
    xg, wg = x.float().cuda().requires_grad_(), w.float().cuda().requires_grad_()
    kr.scaled_linear(xg, wg).backward(d.float().cuda())
    for i, j in ((0, 0), (4, 129), (2, 77)):
        step = torch.zeros_like(x)
        step[i, j] = 1
        assert float(xg.grad[i, j]) == float((((x + step) @ w.t() - (x - step) @ w.t()) * d).sum() / 2)
    for i, j in ((0, 0), (8, 129), (5, 31)):
        step = torch.zeros_like(w)
        step[i, j] = 1
        assert float(wg.grad[i, j]) == float(((x @ (w + step).t() - x @ (w - step).t()) * d).sum() / 2)


def test_linear_without_rows(kr):
    x = torch.zeros(0, 64, device="cuda", requires_grad=True)
    w = torch.ones(40, 64, device="cuda", requires_grad=True)
    kr.scaled_linear(x, w).backward(torch.zeros(0, 40, device="cuda"))
    assert x.grad.shape == (0, 64) and w.grad.shape == (40, 64) and not w.grad.any()


def test_what_has_no_gradient(kr):
    x = make(40, 72, 5).cuda().requires_grad_()
    held = kr.scaled_hold(make(16, 72, 6).cuda(), square=True).plain
    with pytest.raises(ValueError):
        kr.scaled_hold(x)
    with pytest.raises(ValueError):
        kr.scaled_linear(x, held)
    with torch.no_grad():
        assert kr.scaled_linear(x, held).shape == (40, 16)


def test_captured_and_on_another_stream(kr):
    """Forward and backward in one graph, replayed beside eager calls on another stream."""
    x, w, d = make(300, 260, 1).cuda(), make(140, 260, 2).cuda(), make(300, 140, 3).cuda()

    def step():
        return (kr.scaled_linear(x, w), *kr.scaled_linear_backward(d, x, w))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for s in range(4):
        x.copy_(make(300, 260, 10 + s))
        d.copy_(make(300, 140, 20 + s))
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(side):
            want = step()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(p, q) for p, q in zip(got, want)), s
        torch.cuda.synchronize()
