"""Gated projection and its backward pass against the formulas in 64 bits: odd sizes, one row,
strides and alignments, large and small tiles, split sums, infinities and NaN next to and inside
the matrices; gradients also against differences.

Tolerances, all from the formulas.  u = 2^-p is half an ulp of the type (p = 8 bfloat16, 11
float16).  A product over K terms in 32 bits is off by at most (K + 8) 2^-24 sum |a||b|.  The
activation's exponential and reciprocal are taken as 2^-16 relative.  |act'| <= 1.13 for both,
and |act''| <= 1.2 covers the slope's own dependence on g.  dg and du are rounded to the type
between the products, u relative (and 2^-25 where float16 ends)."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
FLOOR = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25}
F32 = 2.0 ** -24
FN = 2.0 ** -16
TYPES = list(U)
SHAPES = [(1, 1, 1), (1, 8, 8), (1, 64, 64), (3, 7, 5), (2, 4096, 1024), (16, 72, 40), (17, 33, 65),
          (31, 520, 96), (33, 2056, 130), (64, 128, 256), (130, 72, 200), (129, 1030, 273),
          (256, 512, 256), (300, 264, 520), (513, 200, 1000), (1000, 64, 16)]
LARGE = [(2048, 136, 4096), (4096, 4096, 72), (200, 4096, 2056)]


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def make(rows, width, hidden, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, width, generator=g).to(dtype)
    wg = (torch.randn(hidden, width, generator=g) * 1.5 / math.sqrt(width)).to(dtype)
    wu = (torch.randn(hidden, width, generator=g) / math.sqrt(width)).to(dtype)
    dh = torch.randn(rows, hidden, generator=g).to(dtype)
    return [t.cuda() for t in (x, wg, wu, dh)]


def act64(g, act):
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p + g * p * (1 - p)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g ** 3))
    return g / 2 * (1 + t), (1 + t) / 2 + g / 2 * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


class Want:
    """Everything in 64 bits, and how far the 32-bit products may be off."""

    def __init__(self, x, wg, wu, dh, act, dtype):
        x, wg, wu, dh = (t.double() for t in (x, wg, wu, dh))
        u = U[dtype]
        rows, width = x.shape
        hidden = wg.shape[0]
        g, up = x @ wg.t(), x @ wu.t()
        eg = (width + 8) * F32 * (x.abs() @ wg.abs().t())
        eu = (width + 8) * F32 * (x.abs() @ wu.abs().t())
        v, s = act64(g, act)
        self.h = v * up
        eh = 1.13 * eg * (up.abs() + eu) + v.abs() * eu + 4 * FN * (v * up).abs()
        self.eh = eh * (1 + u) + u * self.h.abs() + FLOOR[dtype]
        dg, du = dh * up * s, dh * v
        edg = dh.abs() * (eu * 1.13 + (up.abs() + eu) * (1.2 * eg + 8 * FN))
        edg = edg * (1 + u) + u * dg.abs() + FLOOR[dtype]
        edu = dh.abs() * (1.13 * eg + 4 * FN * v.abs())
        edu = edu * (1 + u) + u * du.abs() + FLOOR[dtype]

        def product(a, ea, b, k):
            want = a @ b
            off = ea @ b.abs() + (k + 8) * F32 * ((a.abs() + ea) @ b.abs())
            return want, off

        a, ea = product(dg, edg, wg, 2 * hidden)
        b, eb = product(du, edu, wu, 2 * hidden)
        self.dx, self.edx = a + b, (ea + eb) * (1 + u) + u * (a + b).abs() + FLOOR[dtype]
        self.dwg, e = product(dg.t(), edg.t(), x, rows)
        self.edwg = e * (1 + u) + u * self.dwg.abs() + FLOOR[dtype]
        self.dwu, e = product(du.t(), edu.t(), x, rows)
        self.edwu = e * (1 + u) + u * self.dwu.abs() + FLOOR[dtype]


def near(got, want, off, what):
    d = (got.double() - want).abs()
    assert torch.isfinite(got).all(), what
    assert (d <= off).all(), "%s: %d values, worst %g of the bound" % (
        what, int((d > off).sum()), float((d / off).max()))


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES + LARGE)
def test_forward_and_backward(kr, shape, dtype, act):
    print("gated", shape, dtype, act, flush=True)
    x, wg, wu, dh = make(*shape, dtype, sum(shape))
    w = Want(x, wg, wu, dh, act, dtype)
    near(kr.gated_projection(x, wg, wu, act), w.h, w.eh, "h")
    dx, dwg, dwu = kr.gated_projection_backward(dh, x, wg, wu, act)
    near(dx, w.dx, w.edx, "dx")
    near(dwg, w.dwg, w.edwg, "dwg")
    near(dwu, w.dwu, w.edwu, "dwu")


def test_gradient_against_differences(kr):
    """In float16 with inputs of a few bits: central differences of the formula in 64 bits, the
    step's own error being step^2 times a third derivative of order 1."""
    rows, width, hidden = 5, 6, 7
    x, wg, wu, dh = make(rows, width, hidden, torch.float16, 3)
    for act in ("silu", "gelu"):
        grads = kr.gated_projection_backward(dh, x, wg, wu, act)
        w = Want(x, wg, wu, dh, act, torch.float16)
        args = [t.double() for t in (x, wg, wu)]

        def loss(p):
            g, u = p[0] @ p[1].t(), p[0] @ p[2].t()
            return float((act64(g, act)[0] * u * dh.double()).sum())

        step = 1e-5
        for k, off in enumerate((w.edx, w.edwg, w.edwu)):
            for i in range(args[k].shape[0]):
                for j in range(args[k].shape[1]):
                    hi, lo = [list(args), list(args)]
                    hi[k], lo[k] = args[k].clone(), args[k].clone()
                    hi[k][i, j] += step
                    lo[k][i, j] -= step
                    num = (loss(hi) - loss(lo)) / (2 * step)
                    assert abs(num - float(grads[k][i, j])) <= float(off[i, j]) + 1e-6


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gap,start", [(8, 8), (3, 0), (5, 1), (24, 16)])
def test_strides_and_what_lies_beside(kr, dtype, gap, start):
    """Matrices inside larger ones whose other values are NaN: nothing of them comes in, and
    the results are those of the matrices alone."""
    rows, width, hidden = 133, 200, 152
    x, wg, wu, dh = make(rows, width, hidden, dtype, 8)

    def inside(t):
        big = torch.full((t.shape[0] + 2, t.shape[1] + start + gap), float("nan"), dtype=dtype,
                         device="cuda")
        v = big[1:-1, start:start + t.shape[1]]
        v.copy_(t)
        return v

    a = kr.gated_projection(x, wg, wu)
    b = kr.gated_projection(inside(x), inside(wg), inside(wu))
    assert torch.equal(a, b)
    a = kr.gated_projection_backward(dh, x, wg, wu)
    b = kr.gated_projection_backward(inside(dh), inside(x), inside(wg), inside(wu))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("rows", [1, 9, 32])
def test_few_rows_beside_nan(kr, rows):
    """The same for the form of few rows, which reads the matrices as they lie."""
    for width, hidden, start, gap in ((200, 152, 8, 8), (131, 75, 3, 2), (64, 33, 1, 0)):
        x, wg, wu, _ = make(rows, width, hidden, torch.bfloat16, width)

        def inside(t):
            big = torch.full((t.shape[0] + 2, t.shape[1] + start + gap), float("nan"),
                             dtype=t.dtype, device="cuda")
            v = big[1:-1, start:start + t.shape[1]]
            v.copy_(t)
            return v

        assert torch.equal(kr.gated_projection(inside(x), inside(wg), inside(wu)),
                           kr.gated_projection(x, wg, wu))


@pytest.mark.parametrize("at", [0, 1])
def test_weights_of_unlike_strides(kr, at):
    """One weight matrix inside a larger one, aligned and not, the other by itself."""
    x, wg, wu, dh = make(90, 64, 48, torch.bfloat16, 2)
    want = kr.gated_projection_backward(dh, x, wg, wu)
    for start, gap in ((8, 8), (3, 2)):
        big = torch.full((50, 64 + start + gap), float("nan"), dtype=torch.bfloat16, device="cuda")
        view = big[1:-1, start:start + 64]
        view.copy_((wg, wu)[at])
        w = [wg, wu]
        w[at] = view
        got = kr.gated_projection_backward(dh, x, *w)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        assert torch.equal(kr.gated_projection(x, *w), kr.gated_projection(x, wg, wu))


def test_outputs_inside_larger_matrices(kr):
    """The C entry points write their rows and nothing between them."""
    rows, width, hidden = 70, 40, 52
    x, wg, wu, dh = make(rows, width, hidden, torch.bfloat16, 4)
    want = kr.gated_projection(x, wg, wu)
    grads = kr.gated_projection_backward(dh, x, wg, wu)
    g, _, keep = kr._gated(x, wg, wu, "silu")
    import ctypes

    def room(r, c):
        return torch.full((r, c + 3), 7.0, dtype=torch.bfloat16, device="cuda")

    out = room(rows, hidden)
    wsb = kr._lib.kr_gated_projection_workspace(ctypes.byref(g))
    ws = torch.empty(wsb + 16, dtype=torch.uint8, device="cuda")
    kr._check("f", kr._lib.kr_gated_projection(ctypes.byref(g), kr._ptr(out), hidden + 3,
                                               kr._ptr(ws), wsb, kr._stream()))
    assert torch.equal(out[:, :hidden], want) and (out[:, hidden:] == 7).all()
    outs = [room(rows, width), room(hidden, width), room(hidden, width)]
    wsb = kr._lib.kr_gated_projection_backward_workspace(ctypes.byref(g))
    ws = torch.full((wsb + 64,), 255, dtype=torch.uint8, device="cuda")  # NaN wherever it is read
    kr._check("b", kr._lib.kr_gated_projection_backward(
        ctypes.byref(g), kr._ptr(dh), hidden, kr._ptr(outs[0]), width + 3, kr._ptr(outs[1]),
        width + 3, kr._ptr(outs[2]), width + 3, kr._ptr(ws), wsb, kr._stream()))
    for o, w in zip(outs, grads):
        assert torch.equal(o[:, :width], w) and (o[:, width:] == 7).all()
    assert (ws[wsb:] == 255).all()


@pytest.mark.parametrize("rows", [1, 5, 40, 300])
def test_nan_and_infinity_stay_in_their_rows(kr, rows):
    x, wg, wu, dh = make(rows + 1, 96, 72, torch.bfloat16, rows)
    clean = kr.gated_projection(x, wg, wu)
    x[rows // 2, 5] = float("nan")
    got = kr.gated_projection(x, wg, wu)
    assert got[rows // 2].isnan().all()
    keep = torch.arange(rows + 1) != rows // 2
    assert torch.equal(got[keep], clean[keep])
    dx, dwg, dwu = kr.gated_projection_backward(dh, x, wg, wu)
    assert dx[rows // 2].isnan().all() and dx[keep].isfinite().all()
    assert dwg.isnan().all() and dwu.isnan().all()  # a sum over all rows
    x[rows // 2, 5] = 0
    wg[3, 1] = float("inf")
    got = kr.gated_projection(x, wg, wu)
    cols = torch.arange(72) != 3
    assert not got[:, 3].isfinite().all() and got[:, cols].isfinite().all()


def test_saturated_activations(kr):
    """Gates far out on both sides: act(g) is g or 0, its slope 1 or 0, and nothing overflows."""
    x = torch.ones(4, 8, dtype=torch.float16, device="cuda")
    wu = torch.full((16, 8), 0.5, dtype=torch.float16, device="cuda")
    for big in (100.0, 4000.0):
        wg = torch.full((16, 8), big / 8, dtype=torch.float16, device="cuda")
        wg[::2] *= -1
        dh = torch.ones(4, 16, dtype=torch.float16, device="cuda")
        for act in ("silu", "gelu"):
            h = kr.gated_projection(x, wg, wu, act)
            assert (h[:, ::2] == 0).all() and (h[:, 1::2] == big * 4).all()
            dx, dwg, dwu = kr.gated_projection_backward(dh, x, wg, wu, act)
            assert (dwg[::2] == 0).all() and (dwg[1::2] == 16).all()
            assert (dwu[::2] == 0).all() and (dwu[1::2] == 4 * big).all()


def test_no_rows(kr):
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(24, 64, dtype=torch.bfloat16, device="cuda")
    assert kr.gated_projection(x, w, w).shape == (0, 24)
    dx, dwg, dwu = kr.gated_projection_backward(x[:, :24], x, w, w)
    assert dx.shape == (0, 64) and (dwg == 0).all() and (dwu == 0).all()
    y = torch.zeros(2, 3, 64, dtype=torch.bfloat16, device="cuda")
    assert kr.gated_projection(y, w, w).shape == (2, 3, 24)


def test_same_bits_again_and_on_another_stream(kr):
    x, wg, wu, dh = make(200, 520, 300, torch.bfloat16, 1)
    first = (kr.gated_projection(x, wg, wu),) + kr.gated_projection_backward(dh, x, wg, wu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [(kr.gated_projection(x, wg, wu),) + kr.gated_projection_backward(dh, x, wg, wu)
                 for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    for a in again:
        assert all(torch.equal(p, q) for p, q in zip(a, first))


def test_graph_replays(kr):
    x, wg, wu, dh = make(100, 130, 70, torch.float16, 6)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        kr.gated_projection_backward(dh, x, wg, wu)
        kr.gated_projection(x, wg, wu)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = (kr.gated_projection(x, wg, wu),) + kr.gated_projection_backward(dh, x, wg, wu)
    for k in range(3):
        x.copy_(torch.randn(100, 130, generator=torch.Generator().manual_seed(k)))
        graph.replay()
        torch.cuda.synchronize()
        want = (kr.gated_projection(x, wg, wu),) + kr.gated_projection_backward(dh, x, wg, wu)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
