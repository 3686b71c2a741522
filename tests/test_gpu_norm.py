"""Norm with the residual's addition (forward, 8-bit output, backward) against the same
formulas in 64 bits, on odd widths, strided and unaligned rows, empty batches and rows without
a usable value; gradients also against differences of the forward formula.

Tolerances.  A stored value is rounded once: half an ulp of its type: 2^-p relative, with
p = 8 (bfloat16), 11 (float16) or 24 (float32) bits of significand.  The arithmetic before that is in 32 bits: a sum of squares
over `width` terms added as a tree of short runs is off by at most (longest run + 10) * 2^-24
relative, the longest run being ceil(width / 1024) or 16 terms, so 64 * 2^-24 covers every width
here, and a few roundings of the factor and the products are within it.  A gradient subtracts
two terms: the same bound holds relative to the terms' magnitudes."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25, torch.float32: 1e-37}
WORK = 64 * 2.0 ** -24
TYPES = list(HALF_ULP)
SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 8), (4, 64), (9, 511), (6, 513), (7, 1000), (5, 1024),
          (3, 1025), (4, 2048), (2, 2057), (3, 4097), (2, 8191), (2, 8200), (2, 16384),
          (2, 16385), (2, 40001), (1031, 96)]


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def make(rows, width, dtype, seed, n=4):
    g = torch.Generator().manual_seed(seed)
    got = [torch.randn(rows, width, generator=g).to(dtype) for _ in range(n)]
    return got, (1 + 0.3 * torch.randn(width, generator=g)).to(dtype)


def formula(x, r, w, eps):
    s = x.double() + (r.double() if r is not None else 0)
    f = 1 / (s.square().mean(-1) + eps).sqrt()
    return s, f, s * f[:, None] * w.double()


def near(got, want, size, dtype, what):
    """|got - want| within half an ulp of the value and the arithmetic's share of `size`."""
    d = (got.double().cpu() - want).abs()
    lim = want.abs() * HALF_ULP[dtype] + size * WORK * (1 + HALF_ULP[dtype]) + TINY[dtype]
    bad = d > lim
    assert not bad.any(), "%s: %d values, worst %g of the bound" % (
        what, int(bad.sum()), float((d / lim).max()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", SHAPES)
def test_forward(kr, rows, width, dtype):
    (x, r, _, _), w = make(rows, width, dtype, rows * 7 + width)
    for res in (r, None):
        got = kr.add_rms_norm(x.cuda(), w.cuda(), None if res is None else res.cuda(), eps=1e-5)
        s, f, n = formula(x, res, w, 1e-5)
        near(got.sum, s, s.abs(), dtype, "sum")
        near(got.rstd, f, f, torch.float32, "rstd")
        near(got.out, n, n.abs(), dtype, "norm")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", SHAPES)
def test_bytes(kr, rows, width, dtype):
    (x, r, _, _), w = make(rows, width, dtype, rows * 5 + width)
    got = kr.add_rms_norm_bytes(x.cuda(), w.cuda(), r.cuda(), eps=1e-5)
    s, f, n = formula(x, r, w, 1e-5)
    near(got.sum, s, s.abs(), dtype, "sum")
    near(got.rstd, f, f, torch.float32, "rstd")
    scale = n.abs().amax(-1) / 127
    near(got.scale, scale, scale, torch.float32, "scale")
    q = got.q.cpu()
    assert q.abs().amax(-1).eq(127).all()
    # half a step, and the arithmetic's share of a value that lies between two steps
    off = (q.double() - n / scale[:, None]).abs()
    assert (off <= 0.5 + 127 * 2 * WORK).all(), float(off.max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", SHAPES)
def test_backward(kr, rows, width, dtype):
    (s, g, d, _), w = make(rows, width, dtype, rows * 3 + width)
    f = 1 / (s.double().square().mean(-1) + 1e-5).sqrt()
    f32 = f.float()
    f = f32.double()
    for ds in (d, None):
        dx, dw = kr.add_rms_norm_backward(g.cuda(), s.cuda(), w.cuda(), f32.cuda(),
                                          None if ds is None else ds.cuda())
        h = s.double() * f[:, None]
        gw = g.double() * w.double()
        c = (gw * h).mean(-1, keepdim=True)
        c_size = (gw * h).abs().mean(-1, keepdim=True)
        want = f[:, None] * (gw - h * c) + (ds.double() if ds is not None else 0)
        size = f[:, None] * (gw.abs() + h.abs() * c_size) + (ds.double().abs() if ds is not None
                                                             else 0)
        near(dx, want, size, dtype, "dx")
        # a column's sum: at most rows / 64 terms in a run, 64 and 16 runs in turn
        near(dw, (g.double() * h).sum(0), (g.double() * h).abs().sum(0), torch.float32, "dw")


def test_gradient_against_differences(kr):
    """The gradients of sum(dout * norm) + sum(dsum * s) in float32 against central
    differences of the formula in 64 bits: steps of 1e-4 leave an error of step^2 times the
    third derivative, under 1e-6 here."""
    rows, width, eps = 3, 37, 1e-3
    (x, r, g, d), w = make(rows, width, torch.float32, 11)
    fw = kr.add_rms_norm(x.cuda(), w.cuda(), r.cuda(), eps=eps)
    dx, dw = kr.add_rms_norm_backward(g.cuda(), fw.sum, w.cuda(), fw.rstd, d.cuda())

    def loss(x, w):
        s, _, n = formula(x, r, w, eps)
        return float((n * g.double()).sum() + (s * d.double()).sum())

    step = 1e-4
    for i in range(rows):
        for j in range(0, width, 5):
            e = torch.zeros(rows, width, dtype=torch.float64)
            e[i, j] = step
            num = (loss(x.double() + e, w) - loss(x.double() - e, w)) / (2 * step)
            assert abs(num - float(dx[i, j])) < 2e-5
    for j in range(width):
        e = torch.zeros(width, dtype=torch.float64)
        e[j] = step
        num = (loss(x, w.double() + e) - loss(x, w.double() - e)) / (2 * step)
        assert abs(num - float(dw[j])) < 2e-5


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_alignment_and_shapes(kr, dtype):
    """Rows further apart than they are long, starting off 16 bytes; a 3-D input; columns that
    are not contiguous (copied)."""
    (x, r, _, _), w = make(6, 203, dtype, 5)
    big = torch.zeros(6, 300, dtype=dtype, device="cuda")
    view = big[:, 3:206]
    view.copy_(x.cuda())
    a = kr.add_rms_norm(x.cuda(), w.cuda(), r.cuda())
    b = kr.add_rms_norm(view, w.cuda(), r.cuda())
    assert torch.equal(a.out, b.out) and torch.equal(a.sum, b.sum)
    c = kr.add_rms_norm(x.cuda().reshape(2, 3, 203), w.cuda(), r.cuda().reshape(2, 3, 203))
    assert c.out.shape == (2, 3, 203) and torch.equal(c.out.reshape(6, 203), a.out)
    d = kr.add_rms_norm(x.cuda().t().contiguous().t(), w.cuda(), r.cuda())
    assert torch.equal(d.out, a.out)
    e = kr.add_rms_norm_bytes(view, w.cuda(), r.cuda())
    f = kr.add_rms_norm_bytes(x.cuda(), w.cuda(), r.cuda())
    assert torch.equal(e.q, f.q) and torch.equal(e.scale, f.scale)


def test_in_place(kr):
    """sum over residual and out over x, as a residual stream is kept."""
    for width in (100, 4096, 20000):
        (x, r, _, _), w = make(5, width, torch.bfloat16, width)
        want = kr.add_rms_norm(x.cuda(), w.cuda(), r.cuda())
        xs, rs, ws = x.cuda(), r.cuda(), w.cuda()
        kr._check("kr_add_rms_norm",
                  kr._lib.kr_add_rms_norm(2, 5, width, kr._ptr(xs), width, kr._ptr(rs), width,
                                          kr._ptr(ws), 1e-6, kr._ptr(rs), width, kr._ptr(xs),
                                          width, None, kr._stream()))
        assert torch.equal(xs, want.out) and torch.equal(rs, want.sum)


@pytest.mark.parametrize("over", ["dout", "dsum"])
@pytest.mark.parametrize("width", [100, 1000, 4096, 9000, 16384, 20000])
def test_gradient_in_place(kr, width, over):
    """dx in the place of either gradient that it is made from."""
    (s, g, d, _), w = make(7, width, torch.bfloat16, width)
    f = (1 / s.float().square().mean(-1).sqrt()).cuda()
    s, g, d, w = s.cuda(), g.cuda(), d.cuda(), w.cuda()
    dx, dw = kr.add_rms_norm_backward(g, s, w, f, d)
    got = torch.empty_like(dw)
    wsb = kr._lib.kr_add_rms_norm_backward_workspace(2, 7, width)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    to = g if over == "dout" else d
    kr._check("kr_add_rms_norm_backward",
              kr._lib.kr_add_rms_norm_backward(2, 7, width, kr._ptr(g), width, kr._ptr(s), width,
                                               kr._ptr(w), kr._ptr(f), kr._ptr(d), width,
                                               kr._ptr(to), width, kr._ptr(got), kr._ptr(ws), wsb,
                                               kr._stream()))
    assert torch.equal(to, dx) and torch.equal(got, dw)


@pytest.mark.parametrize("width", [24, 700, 3000, 9000, 20001])
def test_rows_without_a_usable_value(kr, width):
    """Rows of zeros, of values too small for a scale, with a NaN, with an infinity; their
    neighbours are not touched."""
    x = torch.randn(6, width, generator=torch.Generator().manual_seed(1))
    w = torch.ones(width)
    x[1] = 0
    x[2] = 1e-36
    x[3, width // 2] = float("nan")
    x[4, 0] = float("inf")
    got = kr.add_rms_norm_bytes(x.cuda(), w.cuda(), eps=1.0)
    scale, q = got.scale.cpu(), got.q.cpu()
    assert scale[1] == 0 and scale[2] == 0 and scale[3].isnan() and scale[4].isnan()
    assert (q[1:5] == 0).all()
    assert (q[[0, 5]].abs().amax(-1) == 127).all() and scale[[0, 5]].isfinite().all()
    out = kr.add_rms_norm(x.cuda(), w.cuda(), eps=0.0).out.cpu()
    assert out[1].isnan().all()          # 0 / 0: no row factor without eps
    assert out[3].isnan().all()
    assert out[4, 0].isnan() and (out[4, 1:] == 0).all()
    assert out[[0, 5]].isfinite().all()
    zero = kr.add_rms_norm(x.cuda(), w.cuda(), eps=1e-6).out.cpu()
    assert (zero[1] == 0).all()


def test_no_rows(kr):
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    got = kr.add_rms_norm(x, w, x)
    assert got.out.shape == (0, 64) and got.rstd.shape == (0,)
    assert kr.add_rms_norm_bytes(x, w, x).q.shape == (0, 64)
    dx, dw = kr.add_rms_norm_backward(x, x, w, torch.empty(0, device="cuda"))
    assert dx.shape == (0, 64) and (dw == 0).all()


def test_same_bits_again_and_on_another_stream(kr):
    (s, g, d, _), w = make(3000, 1000, torch.bfloat16, 2)
    f = (1 / s.float().square().mean(-1).sqrt()).cuda()
    s, g, d, w = s.cuda(), g.cuda(), d.cuda(), w.cuda()
    first = kr.add_rms_norm_backward(g, s, w, f, d)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [kr.add_rms_norm_backward(g, s, w, f, d) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    for a in again:
        assert torch.equal(a[0], first[0]) and torch.equal(a[1], first[1])


def test_graph_replays(kr):
    (x, r, g, d), w = make(64, 520, torch.float16, 9)
    x, r, g, d, w = x.cuda(), r.cuda(), g.cuda(), d.cuda(), w.cuda()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        fw = kr.add_rms_norm(x, w, r)
        kr.add_rms_norm_backward(g, fw.sum, w, fw.rstd, d)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fw = kr.add_rms_norm(x, w, r)
        dx, dw = kr.add_rms_norm_backward(g, fw.sum, w, fw.rstd, d)
    for k in range(3):
        x.copy_(torch.randn(64, 520, generator=torch.Generator().manual_seed(k)))
        graph.replay()
        torch.cuda.synchronize()
        e = kr.add_rms_norm(x, w, r)
        ex, ew = kr.add_rms_norm_backward(g, e.sum, w, e.rstd, d)
        assert torch.equal(fw.out, e.out) and torch.equal(dx, ex) and torch.equal(dw, ew)
