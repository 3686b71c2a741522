"""Dropout: the mask against the generator written out in whole numbers, values against the formula in
64 bits.

Tolerances.  A kept value is multiplied by the factor (itself rounded to 32 bits), the residual
added, each a rounding of 2^-24 relative to its result, and the sum is rounded to its type: half a
step, eps / 2.  3 * 2^-24 of the terms' sizes covers the 32-bit part."""

import pytest
import torch

from tests.philox import factor

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
SHAPES = [(1, 1), (1, 7), (5, 8), (3, 9), (300, 17), (2, 2048), (7, 2049), (3, 4100), (1, 70001),
          (1031, 96), (4099, 3)]


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def normal(*shape, seed, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def near(got, want, size):
    half = torch.finfo(got.dtype).eps / 2
    off = (got.double().cpu() - want).abs()
    lim = want.abs() * half + size * 3 * 2.0 ** -24 * (1 + half)
    lim = lim + (2.0 ** -25 if got.dtype == torch.float16 else 0)
    assert (off <= lim).all(), float((off - lim).max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", SHAPES)
def test_values(kr, rows, width, dtype):
    x, r = normal(rows, width, seed=1, dtype=dtype), normal(rows, width, seed=2, dtype=dtype)
    for p, seed, offset in ((0.1, 0, 0), (0.5, 2 ** 64 - 1, 2 ** 64 - 1), (0.75, 12345678901234, 7)):
        f = factor(rows, width, p, seed, offset)
        got = kr.dropout(x.cuda(), p, seed, offset)
        assert torch.equal(got.cpu() == 0, (f == 0) | (x == 0))
        near(got, x.double() * f, (x.double() * f).abs())
        got = kr.dropout(x.cuda(), p, seed, offset, r.cuda())
        near(got, x.double() * f + r.double(), (x.double() * f).abs() + r.double().abs())


@pytest.mark.parametrize("dtype", TYPES)
def test_none_and_all(kr, dtype):
    x = normal(9, 300, seed=3, dtype=dtype).cuda()
    r = normal(9, 300, seed=4, dtype=dtype).cuda()
    assert torch.equal(kr.dropout(x, 0.0, 5), x)
    assert torch.equal(kr.dropout(x, 2.0 ** -18, 5), x)  # rounds to no value of 65,536
    assert not kr.dropout(x, 1.0, 5).any()
    assert torch.equal(kr.dropout(x, 1.0, 5, 0, r), r)
    assert kr.dropout(x[:0], 0.5, 5).shape == (0, 300)


def test_dropped_values_are_zero_whatever_they_were(kr):
    f = factor(40, 100, 0.5, 9, 0)
    for bad in (float("nan"), float("inf"), float("-inf")):
        got = kr.dropout(torch.full((40, 100), bad).cuda(), 0.5, 9).cpu()
        assert torch.equal(got == 0, f == 0) and not torch.isfinite(got[f > 0]).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_places(kr, dtype):
    """Rows apart, unaligned starts, crossed and repeated tensors, more dimensions: the mask goes by a
    value's place in the tensor; what lies between rows stays."""
    store = normal(20, 137, seed=5, dtype=dtype).cuda()
    f = factor(20, 131, 0.4, 3, 1)
    for x in (store[:, 1:132], store[:, 6:137], normal(131, 20, seed=6, dtype=dtype).cuda().t(),
              normal(1, 131, seed=7, dtype=dtype).cuda().expand(20, 131)):
        near(kr.dropout(x, 0.4, 3, 1), x.double().cpu() * f, (x.double().cpu() * f).abs())
    x = normal(4, 5, 131, seed=8, dtype=dtype).cuda()
    near(kr.dropout(x, 0.4, 3, 1).reshape(20, 131), x.double().cpu().reshape(20, 131) * f,
         (x.double().cpu().reshape(20, 131) * f).abs())


def test_in_place_and_gaps(kr):
    """The C call on rows apart, onto its input and onto the residual: the gaps keep what they held."""
    import ctypes

    L = kr._lib
    d = kr.KrDrop(0.4, 3, 1, None)
    f = factor(20, 131, 0.4, 3, 1)
    for onto in (0, 1):
        s = [normal(20, 160, seed=9 + k).cuda() for k in range(2)]
        was = [t.clone() for t in s]
        ptr = [t.data_ptr() + 4 for t in s]
        assert L.kr_dropout(kr._TYPES[torch.float32], 20, 131, ptr[0], 160, ptr[1], 160,
                            ctypes.byref(d), ptr[onto], 160, kr._raw_stream(0)) == kr.KR_OK
        assert torch.equal(s[1 - onto], was[1 - onto])
        assert torch.equal(s[onto][:, 132:], was[onto][:, 132:])
        assert torch.equal(s[onto][:, 0], was[onto][:, 0])
        x, r = (t[:, 1:132].double().cpu() for t in was)
        near(s[onto][:, 1:132], x * f + r, (x * f).abs() + r.abs())


def test_rows_past_one_launch(kr):
    """More rows than one grid takes (2^23 blocks, one row each), past 32-bit offsets: the counters go
    on."""
    edge, width = 1 << 23, 1032
    x = torch.ones(edge + 9, width, dtype=torch.bfloat16, device="cuda")
    got = kr.dropout(x, 0.5, 11, 5)
    for row0 in (0, (1 << 22) - 4, edge - 8, edge + 1):
        f = factor(8, width, 0.5, 11, 5, row0)
        assert torch.equal(got[row0:row0 + 8].double().cpu(), f), row0


def test_gradient(kr):
    x = normal(6, 70, seed=1).cuda().requires_grad_()
    r = normal(6, 70, seed=2).cuda().requires_grad_()
    d = normal(6, 70, seed=3).cuda()
    y = kr.dropout(x, 0.3, 17, 2, r)
    y.backward(d)
    f = factor(6, 70, 0.3, 17, 2)
    near(x.grad, d.double().cpu() * f, (d.double().cpu() * f).abs())
    assert torch.equal(r.grad, d)
    # against differences: D is linear, so a step of 1 shows its gradient
    step = torch.zeros(6, 70).cuda()
    step[2, 5:50] = 1
    with torch.no_grad():
        moved = kr.dropout(step, 0.3, 17, 2)
    near(moved, f * step.double().cpu(), f)
    x.grad = None
    kr.dropout(x, 0.3, 17, 2).sum().backward()
    near(x.grad, f, f)


def test_seed_on_the_device(kr):
    x = normal(30, 70, seed=1).cuda()
    for value in (0, 5, -1):
        seed = torch.tensor([value], device="cuda")
        assert torch.equal(kr.dropout(x, 0.3, seed, 2), kr.dropout(x, 0.3, value % 2 ** 64, 2))
    # changed between the passes: the backward pass says so
    y = kr.dropout(x.clone().requires_grad_(), 0.3, seed, 2)
    seed += 1
    with pytest.raises(RuntimeError):
        y.sum().backward()


def test_captured(kr):
    """A captured call, replayed with new inputs and new seeds, beside eager calls."""
    x = normal(64, 200, seed=1).cuda()
    seed = torch.zeros(1, dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kr.dropout(x, 0.3, seed, 2)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = kr.dropout(x, 0.3, seed, 2)
    for k in range(4):
        seed.fill_(100 + k)
        x.copy_(normal(64, 200, seed=10 + k))
        graph.replay()
        assert torch.equal(y, kr.dropout(x, 0.3, 100 + k, 2)), k
        torch.cuda.synchronize()
