"""Layer norm with the residual's addition and dropout, forward and backward, against the formulas in
64 bits: odd widths, strided and unaligned rows, empty batches, rows of one value, rows far from
zero; gradients also against differences.

Tolerances.  A stored value is rounded once, half a step: eps / 2 of its type.  The arithmetic
before that is in 32 bits.  A sum over a row's terms, added as a tree of runs of at most 64, is off by
at most WORK = 64 * 2^-24 of the terms' sizes (a run of up to ceil(width / 1024) or 16, 10 steps between
threads, and a few roundings).  Forward, with S a row's largest |D(x)| + |r|: s and its mean are off by
WORK S together, so a difference from the mean by E = 2 WORK S, and the factor, of differences each off by E,
by WORK + E f relative (the mean square of differences off by E is off by 2 E sqrt(v) + E^2, and the factor
by half of that over v; f <= 1 / sqrt(v)), E f < 1/4.  Backward, s, mean and rstd are inputs: terms are off by
WORK of their sizes."""

import pytest
import torch

from tests.philox import factor

pytestmark = pytest.mark.gpu

TINY = {torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25, torch.float32: 1e-37}
WORK = 64 * 2.0 ** -24
TYPES = list(TINY)
SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 8), (4, 64), (9, 511), (6, 513), (7, 1000), (5, 1024),
          (3, 1025), (4, 2048), (2, 2057), (3, 4097), (2, 8191), (2, 8200), (2, 16384),
          (2, 16385), (2, 40001), (1031, 96)]
DROP = dict(p=0.3, seed=77, offset=5)


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def make(rows, width, dtype, seed, n=4):
    g = torch.Generator().manual_seed(seed)
    got = [torch.randn(rows, width, generator=g).to(dtype) for _ in range(n)]
    return got, (1 + 0.3 * torch.randn(width, generator=g)).to(dtype), \
        (0.3 * torch.randn(width, generator=g)).to(dtype)


def near(got, want, off, dtype, what):
    """|got - want| within half a step of the value and the arithmetic's share `off`."""
    half = torch.finfo(dtype).eps / 2
    d = (got.double().cpu() - want).abs()
    lim = want.abs() * half + off * (1 + half) + TINY[dtype]
    bad = ~(d <= lim)
    assert not bad.any(), "%s: %d values, worst %g of the bound" % (
        what, int(bad.sum()), float((d / lim).max()))


def check_forward(got, x, r, w, b, eps, f, dtype):
    branch = x.double() * f
    res = r.double() if r is not None else torch.zeros_like(branch)
    s = branch + res
    top = (branch.abs() + res.abs()).amax(-1, keepdim=True)
    m = s.mean(-1, keepdim=True)
    rstd = 1 / ((s - m).square().mean(-1, keepdim=True) + eps).sqrt()
    e = 2 * WORK * top
    assert (e * rstd < 0.25).all()
    rel = WORK + e * rstd * 1.5  # E f, and what its square adds below 1/4
    near(got.sum, s, WORK * (branch.abs() + res.abs()), dtype, "sum")
    near(got.mean, m[:, 0], (WORK * top)[:, 0], torch.float32, "mean")
    near(got.rstd, rstd[:, 0], (rel * rstd)[:, 0], torch.float32, "rstd")
    h = (s - m) * rstd
    bias = b.double() if b is not None else torch.zeros_like(w.double())
    off = (h.abs() * rel + e * rstd * (1 + rel)) * w.double().abs() * (1 + WORK)
    near(got.out, h * w.double() + bias, off + WORK * ((h * w.double()).abs() + bias.abs()), dtype,
         "norm")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", SHAPES)
def test_forward(kr, rows, width, dtype):
    (x, r, _, _), w, b = make(rows, width, dtype, rows * 7 + width)
    f = factor(rows, width, DROP["p"], DROP["seed"], DROP["offset"])
    for res, bias, drop in ((r, b, {}), (None, b, {}), (r, None, DROP), (None, b, DROP)):
        got = kr.add_layer_norm(x.cuda(), w.cuda(), None if bias is None else bias.cuda(),
                                None if res is None else res.cuda(), eps=1e-3, **drop)
        check_forward(got, x, res, w, bias, 1e-3, f if drop else 1.0, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", SHAPES)
def test_backward(kr, rows, width, dtype):
    (s, g, d, _), w, _ = make(rows, width, dtype, rows * 3 + width)
    mean = s.double().mean(-1).float()
    rstd = (1 / ((s.double() - mean.double()[:, None]).square().mean(-1) + 1e-3).sqrt()).float()
    f = factor(rows, width, DROP["p"], DROP["seed"], DROP["offset"])
    for ds, drop in ((d, {}), (None, DROP), (d, DROP)):
        dx, dres, dw, db = kr.add_layer_norm_backward(
            g.cuda(), s.cuda(), w.cuda(), mean.cuda(), rstd.cuda(),
            None if ds is None else ds.cuda(), **drop)
        a = rstd.double()[:, None]
        h = (s.double() - mean.double()[:, None]) * a
        t = g.double() * w.double()
        more = ds.double() if ds is not None else torch.zeros_like(h)
        want = a * (t - t.mean(-1, keepdim=True) - h * (t * h).mean(-1, keepdim=True)) + more
        size = a * (t.abs() + t.abs().mean(-1, keepdim=True) +
                    h.abs() * (t * h).abs().mean(-1, keepdim=True)) + more.abs()
        near(dres, want, WORK * size, dtype, "dresidual")
        if drop:
            near(dx, want * f, WORK * size * f, dtype, "dx")
            assert not dx.cpu()[f == 0].any()
        else:
            assert dx is dres
        # a column's sum: at most rows / 64 terms in a run, 64 and 16 runs in turn
        near(dw, (g.double() * h).sum(0), WORK * (g.double() * h).abs().sum(0), torch.float32, "dw")
        near(db, g.double().sum(0), WORK * g.double().abs().sum(0), torch.float32, "db")


def test_gradient_against_differences(kr):
    """The gradients of sum(dout * norm) + sum(dsum * s) in float32 against central differences of the
    formula in 64 bits: steps of 1e-4 leave an error of step^2 times the third derivative, under 1e-6
    here."""
    rows, width, eps = 3, 37, 1e-2
    (x, r, g, d), w, b = make(rows, width, torch.float32, 11)
    f = factor(rows, width, DROP["p"], DROP["seed"], DROP["offset"])
    fw = kr.add_layer_norm(x.cuda(), w.cuda(), b.cuda(), r.cuda(), eps=eps, **DROP)
    grads = kr.add_layer_norm_backward(g.cuda(), fw.sum, w.cuda(), fw.mean, fw.rstd, d.cuda(), **DROP)

    def loss(x, r, w, b):
        s = x * f + r
        c = s - s.mean(-1, keepdim=True)
        n = c / (c.square().mean(-1, keepdim=True) + eps).sqrt() * w + b
        return float((n * g.double()).sum() + (s * d.double()).sum())

    at = [t.double() for t in (x, r, w, b)]
    step = 1e-4
    for k, grad in enumerate(grads):
        flat = at[k].view(-1)
        for i in range(0, flat.numel(), 7):
            keep = float(flat[i])
            flat[i] = keep + step
            up = loss(*at)
            flat[i] = keep - step
            down = loss(*at)
            flat[i] = keep
            want = (up - down) / (2 * step)
            # 32-bit arithmetic on sums of some 40 terms of size up to 10
            assert abs(float(grad.view(-1)[i]) - want) <= 1e-6 + 40 * 10 * WORK / 8, (k, i)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_far_from_zero_and_of_one_value(kr, dtype):
    """The variance is that of the differences: rows about 100 with deviations of 1 keep theirs."""
    (x, r, _, _), w, b = make(5, 1000, dtype, 3)
    r = (r.double() + 100).to(dtype)
    got = kr.add_layer_norm(x.cuda(), w.cuda(), b.cuda(), r.cuda(), eps=1e-3)
    check_forward(got, x, r, w, b, 1e-3, 1.0, dtype)
    same = torch.full((3, 700), 2.5, dtype=dtype)
    got = kr.add_layer_norm(same.cuda(), w[:700].cuda(), b[:700].cuda())
    assert torch.equal(got.out.cpu(), b[:700].expand(3, 700)) and (got.mean == 2.5).all()
    near(got.rstd, torch.full((3,), 1e-5 ** -0.5, dtype=torch.float64), 1e-5 ** -0.5 * WORK,
         torch.float32, "rstd")


@pytest.mark.parametrize("width", [96, 1000, 5000, 16384, 20000])
def test_bad_rows_stay_alone(kr, width):
    """A NaN or infinity spoils its own row of the outputs and nothing of others; dropped, it spoils
    nothing."""
    (x, r, g, d), w, b = make(6, width, torch.float32, 5)
    x[2, width // 3] = float("nan")
    x[4, width - 1] = float("inf")
    clean = x.clone()
    clean[2], clean[4] = 0, 0
    for bad in (False, True):
        got = kr.add_layer_norm((x if bad else clean).cuda(), w.cuda(), b.cuda(), r.cuda())
        if not bad:
            good = got
    keep = [0, 1, 3, 5]
    assert torch.equal(got.out[keep], good.out[keep]) and got.out[[2, 4]].isnan().all()
    f = factor(6, width, 0.5, 0, 0)
    x = torch.where(f.float() == 0, torch.full_like(x, float("nan")), clean)
    zero = torch.where(f.float() == 0, torch.zeros_like(x), clean)
    one = kr.add_layer_norm(x.cuda(), w.cuda(), b.cuda(), r.cuda(), p=0.5)
    two = kr.add_layer_norm(zero.cuda(), w.cuda(), b.cuda(), r.cuda(), p=0.5)
    assert torch.equal(one.out, two.out) and torch.equal(one.sum, two.sum)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [33, 515, 2057, 4099])
def test_strided_rows(kr, width, dtype):
    """Rows apart, from unaligned addresses, between NaN: as from contiguous ones."""
    (x, r, g, d), w, b = make(7, width, dtype, 9)

    def wide(t):
        store = torch.full((7, width + 5), float("nan"), dtype=dtype).cuda()
        store[:, 3:3 + width] = t.cuda()
        return store[:, 3:3 + width]

    one = kr.add_layer_norm(x.cuda(), w.cuda(), b.cuda(), r.cuda(), **DROP)
    two = kr.add_layer_norm(wide(x), w.cuda(), b.cuda(), wide(r), **DROP)
    for k in ("out", "sum", "mean", "rstd"):
        assert torch.equal(getattr(one, k), getattr(two, k)), k
    one = kr.add_layer_norm_backward(g.cuda(), one.sum, w.cuda(), one.mean, one.rstd, d.cuda(), **DROP)
    two = kr.add_layer_norm_backward(wide(g), wide(two.sum.cpu()), w.cuda(), two.mean, two.rstd,
                                     wide(d), **DROP)
    assert all(torch.equal(p, q) for p, q in zip(one, two))


@pytest.mark.parametrize("width", [65, 2000, 9000, 17000])
def test_outputs_in_place_and_between_marks(kr, width):
    """sum over x and out over the residual; gradients over dout and dsum; gaps between rows keep what
    they held."""
    import ctypes

    L, t, st = kr._lib, kr._TYPES[torch.float32], kr._raw_stream(0)
    (x, r, g, d), w, b = (v.cuda() if isinstance(v, torch.Tensor) else [u.cuda() for u in v]
                          for v in make(5, width, torch.float32, 4))
    drop = kr.KrDrop(0.3, 77, 5, None)
    n = kr.add_layer_norm(x, w, b, r, eps=1e-3, **DROP)
    ld = width + 9
    store = [torch.full((5, ld), 7.0, device="cuda") for _ in range(4)]
    for s, v in zip(store, (x, r, g, d)):
        s[:, :width] = v
    mean, rstd = torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    at = [s.data_ptr() for s in store]
    assert L.kr_add_layer_norm(t, 5, width, at[0], ld, at[1], ld, w.data_ptr(), b.data_ptr(), 1e-3,
                               ctypes.byref(drop), at[0], ld, at[1], ld, mean.data_ptr(),
                               rstd.data_ptr(), st) == 0
    assert torch.equal(store[0][:, :width], n.sum) and torch.equal(store[1][:, :width], n.out)
    back = kr.add_layer_norm_backward(g, n.sum, w, mean, rstd, d, **DROP)
    dw, db = torch.empty(width, device="cuda"), torch.empty(width, device="cuda")
    wsb = L.kr_add_layer_norm_backward_workspace(t, 5, width)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    assert L.kr_add_layer_norm_backward(t, 5, width, at[2], ld, at[0], ld, w.data_ptr(),
                                        mean.data_ptr(), rstd.data_ptr(), at[3], ld,
                                        ctypes.byref(drop), at[2], ld, at[3], ld, dw.data_ptr(),
                                        db.data_ptr(), ws.data_ptr(), wsb, st) == 0
    for got, want in zip((store[3][:, :width], store[2][:, :width], dw, db), back):
        assert torch.equal(got, want)
    assert all((s[:, width:] == 7).all() for s in store)


def test_empty_and_many_rows(kr):
    w, b = torch.ones(96).cuda(), torch.zeros(96).cuda()
    x = torch.zeros(0, 96).cuda()
    got = kr.add_layer_norm(x, w, b, x, p=0.1)
    assert got.out.shape == (0, 96) and got.mean.shape == (0,)
    dx, dres, dw, db = kr.add_layer_norm_backward(x, x, w, got.mean, got.rstd)
    assert not dw.any() and not db.any() and dx.shape == (0, 96)
    # more rows than one launch takes: the counters of dropout go on
    n = (1 << 21) + 50
    x = torch.ones(n, 8, device="cuda").half()
    x[:, 1::2] = 2
    got = kr.add_layer_norm(x, w[:8].half(), p=0.5, seed=3, offset=1)
    for row0 in (0, (1 << 21) - 8, n - 16):
        f = factor(16, 8, 0.5, 3, 1, row0)
        assert torch.equal(got.sum[row0:row0 + 16].double().cpu(),
                           x[row0:row0 + 16].double().cpu() * f)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_autograd(kr, dtype, p):
    (x, r, g, d), w, b = make(10, 72, dtype, 8)
    x, r, w, b = (v.reshape(2, 5, 72) if v.dim() == 2 else v for v in (x, r, w, b))
    x, r, w, b = (v.cuda().requires_grad_() for v in (x, r, w, b))
    g, d = g.reshape(2, 5, 72).cuda(), d.reshape(2, 5, 72).cuda()
    drop = dict(p=p, seed=4, offset=9)
    n = kr.add_layer_norm(x, w, b, r, **drop)
    assert n.out.requires_grad and n.sum.requires_grad
    assert not n.mean.requires_grad and not n.rstd.requires_grad
    torch.autograd.backward([n.out, n.sum], [g, d])
    with torch.no_grad():
        m = kr.add_layer_norm(x, w, b, r, **drop)
        assert all(torch.equal(getattr(m, k), getattr(n, k)) for k in ("out", "sum", "mean", "rstd"))
        dx, dres, dw, db = kr.add_layer_norm_backward(g, m.sum, w, m.mean, m.rstd, d, **drop)
    assert torch.equal(x.grad, dx) and torch.equal(r.grad, dres)
    assert torch.equal(w.grad, dw.to(dtype)) and torch.equal(b.grad, db.to(dtype))
    # only the sum; only the norm, without residual and bias
    x.grad = r.grad = w.grad = b.grad = None
    kr.add_layer_norm(x, w, b, r, **drop).sum.backward(d)
    assert torch.equal(r.grad, d) and torch.equal(x.grad, kr.dropout(d, p, 4, 9))
    x.grad = None
    n = kr.add_layer_norm(x, w, **drop)
    assert (n.sum is x) == (p == 0)
    n.out.backward(g)
    dx, _, dw, _ = kr.add_layer_norm_backward(g, n.sum.detach(), w.detach(), n.mean, n.rstd, **drop)
    assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw.to(dtype))


def test_captured(kr):
    """Forward and backward in one graph, replayed with new inputs and seeds, beside eager calls."""
    (x, r, g, d), w, b = make(300, 520, torch.bfloat16, 8)
    x, r, g, d, w, b = (v.cuda() for v in (x, r, g, d, w, b))
    seed = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step():
        n = kr.add_layer_norm(x, w, b, r, p=0.2, seed=seed)
        return (n.out, n.sum) + kr.add_layer_norm_backward(g, n.sum, w, n.mean, n.rstd, d, p=0.2,
                                                           seed=seed)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(4):
        seed.fill_(k)
        (a, c, _, _), _, _ = make(300, 520, torch.bfloat16, 20 + k)
        x.copy_(a)
        r.copy_(c)
        graph.replay()
        want = step()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), k
        torch.cuda.synchronize()


def test_past_32_bit_offsets(kr):
    """More than 2^32 elements, rows of a repeated pattern: forward and backward as from the pattern alone, but
    for the sums over rows, which are the pattern's many times."""
    part, w, b = make(64, 2100, torch.bfloat16, 12)
    n = 64 * 33000
    x, g = (v.cuda().repeat(n // 64, 1) for v in part[:2])
    w, b = w.cuda(), b.cuda()
    small = kr.add_layer_norm(x[:64], w, b)
    got = kr.add_layer_norm(x, w, b)
    for row0 in (0, n // 2 - 32, n - 64):
        row0 = row0 // 64 * 64
        assert torch.equal(got.out[row0:row0 + 64], small.out)
        assert torch.equal(got.rstd[row0:row0 + 64], small.rstd)
    del got.out
    few = kr.add_layer_norm_backward(g[:64], x[:64], w, small.mean, small.rstd)
    many = kr.add_layer_norm_backward(g, x, w, got.mean, got.rstd)
    for row0 in (0, n // 2 // 64 * 64, n - 64):
        assert torch.equal(many[1][row0:row0 + 64], few[1])
    # A sum of n terms in 32 bits, each added to what there is, is off by at most n 2^-24 of the terms' sizes
    # together (and by n^2 2^-48: the 1.01).  Here a block, one row at a time at this width, adds
    # rows / blocks of them, its share goes into one of 32 runs of blocks / 32, and these are added; h and
    # the product are 4 roundings.  The few rows' sums are off by WORK.
    from paper_2601_17654_amd.binding import _lib, _TYPES

    blocks = _lib.kr_add_layer_norm_backward_workspace(_TYPES[torch.bfloat16], n, 2100) // (8 * 2100)
    adds = -(-n // blocks) + -(-blocks // 32) + 32 + 4
    gd = g[:64].double()
    h = (x[:64].double() - small.mean.double()[:, None]) * small.rstd.double()[:, None]
    for k, size in ((2, (gd * h).abs().sum(0)), (3, gd.abs().sum(0))):
        off = (many[k].double() - few[k].double() * (n // 64)).abs()
        assert (off <= (adds * 2.0 ** -24 + WORK) * 1.01 * size * (n // 64)).all()


def test_past_32_bit_offsets_every_row(kr):
    """The same size with whole numbers of at most 2 for h, dout and weight: sums over rows are whole numbers below
    2^24, exact in any order, so that a row left out or taken twice shows."""
    gen = torch.Generator().manual_seed(13)
    n = 64 * 33000
    s, g = (torch.randint(-2, 3, (64, 2100), generator=gen).to(torch.bfloat16) for _ in range(2))
    assert ((s * g).double().abs().sum(0) * (n // 64) < 2 ** 24).all()
    want = [(s.double() * g.double()).sum(0) * (n // 64), g.double().sum(0) * (n // 64)]
    s, g = (v.cuda().repeat(n // 64, 1) for v in (s, g))
    # the last row alone, past 2^32 elements, differs
    want[0] += (2 - s[-1].double().cpu()) * g[-1].double().cpu()
    s[-1] = 2
    stats = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    w = torch.ones(2100, dtype=torch.bfloat16, device="cuda")
    _, _, dw, db = kr.add_layer_norm_backward(g, s, w, *stats)
    assert torch.equal(dw.double().cpu(), want[0]) and torch.equal(db.double().cpu(), want[1])
