"""Gradients of the gated projection where the output's gradient is far from unit size, as that of
a mean loss is: dg and du, which stand in 16 bits between the products, keep their precision.

In float16 dh is taken times a power of two s, so that its largest magnitude lies in [2^-2, 2^7);
within that range s is 1.  Tolerances are those of the unit-sized test (`Want`) for the
gradient dh s, divided by s, and half of float16's least step for the stored result."""

import math

import pytest
import torch

from tests.test_gpu_gated import F32, Want, act64, make, near

pytestmark = pytest.mark.gpu

LEAST = {torch.float16: 2.0 ** -25, torch.bfloat16: 1e-38}


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def scale_of(dh):
    e = math.floor(math.log2(float(dh.abs()[dh.isfinite()].max())))
    return 2.0 ** (-2 - e) if e < -2 else 2.0 ** (6 - e) if e > 6 else 1.0


def check(kr, x, wg, wu, dh, act, dtype):
    s = scale_of(dh) if dtype == torch.float16 else 1.0
    w = Want(x, wg, wu, dh.double() * s, act, dtype)
    got = kr.gated_projection_backward(dh, x, wg, wu, act)
    for g, want, off, what in zip(got, (w.dx, w.dwg, w.dwu), (w.edx, w.edwg, w.edwu),
                                  ("dx", "dwg", "dwu")):
        near(g, want / s, off / s + LEAST[dtype], what)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("power", [-20, -17, -12, -4, 3])
@pytest.mark.parametrize("shape", [(1, 64, 64), (3, 7, 5), (4, 200, 130), (300, 264, 520)])
def test_sizes(kr, shape, power, dtype, act):
    print("sizes", shape, power, dtype, act, flush=True)
    x, wg, wu, dh = make(*shape, dtype, sum(shape) - power)
    # large x, small weights: the weights' gradients are far above float16's least value
    x, wg, wu = x * 64, wg / 64, wu / 64
    check(kr, x, wg, wu, dh * 2.0 ** power, act, dtype)


@pytest.mark.parametrize("shape", [(9, 200, 16), (70, 64, 24)])
def test_large(kr, shape):
    """dg above float16's range: results within it are as the formula's, those above infinite."""
    x, wg, wu, dh = make(*shape, torch.float16, 5)
    x, wg, wu, dh = x / 16, wg * 16, wu * 128, dh * 2.0 ** 12
    s = scale_of(dh)
    w = Want(x, wg, wu, dh.double() * s, "silu", torch.float16)
    got = kr.gated_projection_backward(dh, x, wg, wu, "silu")
    for g, want, off, what in zip(got, (w.dx, w.dwg, w.dwu), (w.edx, w.edwg, w.edwu),
                                  ("dx", "dwg", "dwu")):
        g, want, off = g.double(), want / s, off / s + LEAST[torch.float16]
        above, below = want.abs() - off >= 65520, want.abs() + off < 65520
        assert not g.isnan().any() and below.any(), what
        assert (g[above] == want[above].sign() * math.inf).all(), what
        assert ((g - want).abs() <= off)[below].all(), what


@pytest.mark.parametrize("power", [-12, -14, -16])
@pytest.mark.parametrize("rows,width,hidden", [(512, 128, 256), (40, 72, 56), (1111, 264, 130)])
def test_small_is_the_unit_one_scaled(kr, rows, width, hidden, power):
    """dh of four bits, so that dh 2^power is exact.  The two calls hold dg and du at sizes a
    power of two apart, the smaller at half the larger's or above: they differ by half a least
    step of the smaller, 2^-24 of the unit call's, and the stored results by their own rounding."""
    x, wg, wu, _ = make(rows, width, hidden, torch.float16, rows)
    x, wg, wu = x * 64, wg / 64, wu / 64
    gen = torch.Generator().manual_seed(power + 100)
    dh = (torch.randint(-8, 9, (rows, hidden), generator=gen) / 16).half().cuda()
    assert float(dh.abs().max()) == 0.5
    unit = kr.gated_projection_backward(dh, x, wg, wu)
    small = kr.gated_projection_backward(dh * 2.0 ** power, x, wg, wu)
    x64, g64, u64 = x.double(), wg.double(), wu.double()
    a, s = act64(x64 @ g64.t(), "silu")
    dg, du = (dh.double() * (x64 @ u64.t()) * s).abs(), (dh.double() * a).abs()
    one = torch.ones_like(dg)

    def bound(p, q, k):
        return 2.0 ** -24 * (one if p.shape == one.shape else one.t()) @ q.abs() \
            + 2.01 * (k + 8) * F32 * (p @ q.abs())

    lims = (bound(dg, g64, 2 * hidden) + bound(du, u64, 2 * hidden), bound(dg.t(), x64, rows),
            bound(du.t(), x64, rows))
    for u, v, lim, what in zip(unit, small, lims, ("dx", "dwg", "dwu")):
        u, v = u.double(), v.double() * 2.0 ** -power
        lim = lim + 2.0 ** -11 * (u.abs() + v.abs()) + 2.0 ** -25 * (1 + 2.0 ** -power)
        d = (u - v).abs()
        assert (d <= lim).all(), "%s: %d values, worst %g of the bound" % (
            what, int((d > lim).sum()), float((d / lim).max()))


def test_values_that_are_no_size(kr):
    """The scale comes from the finite values: a NaN or an infinity in dh stays in its row of dx
    and its column of the weights, all else is as without it; an all-zero dh gives zeros."""
    x, wg, wu, dh = make(130, 96, 72, torch.float16, 9)
    dh = dh * 2.0 ** -15
    dh[7, 5] = 0
    clean = kr.gated_projection_backward(dh, x, wg, wu)
    for bad in (float("nan"), float("inf")):
        dh[7, 5] = bad
        dx, dwg, dwu = kr.gated_projection_backward(dh, x, wg, wu)
        rows, cols = torch.arange(130) != 7, torch.arange(72) != 5
        assert torch.equal(dx[rows], clean[0][rows]) and not dx[7].isfinite().any()
        assert torch.equal(dwg[cols], clean[1][cols]) and not dwg[5].isfinite().any()
        assert torch.equal(dwu[cols], clean[2][cols]) and not dwu[5].isfinite().any()
    for g in kr.gated_projection_backward(torch.zeros_like(dh), x, wg, wu):
        assert (g == 0).all()


@pytest.mark.parametrize("gap,start", [(8, 8), (3, 1)])
def test_a_strided_gradient(kr, gap, start):
    """What lies between dh's rows is no part of its size."""
    x, wg, wu, dh = make(133, 200, 149, torch.float16, 8)
    dh = dh * 2.0 ** -14
    big = torch.full((135, 149 + start + gap), 1000.0, dtype=torch.float16, device="cuda")
    view = big[1:-1, start:start + 149]
    view.copy_(dh)
    a, b = (kr.gated_projection_backward(d, x, wg, wu) for d in (dh, view))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("shape", [(40, 96, 2200), (33, 6000, 40)])
def test_split_sums(kr, shape):
    """Sums that are cut into parts and joined (many terms, few outputs)."""
    x, wg, wu, dh = make(*shape, torch.float16, 3)
    check(kr, x, wg, wu, dh * 2.0 ** -14, "silu", torch.float16)
