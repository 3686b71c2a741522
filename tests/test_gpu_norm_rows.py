"""Norm on rows inside larger matrices.

What lies beside a row is NaN (inputs) or a mark (outputs), so that an element read past a row's end
shows in the sums and one written there shows as a lost mark.  One width for each path: rows
of fewer elements than a vector, several rows a block, one row a block, 16 elements a thread, and
rows that are read again from memory.  Strided and unaligned calls take the same sums in the
same order as contiguous ones: results are equal bit for bit."""

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
CODE = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
WIDTHS = [1, 3, 101, 500, 1003, 2057, 9001, 16390, 20003]
ROWS = 9


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def make(width, dtype, n):
    g = torch.Generator().manual_seed(width)
    return [torch.randn(ROWS, width, generator=g).to(dtype).cuda() for _ in range(n)], (
        1 + 0.3 * torch.randn(width, generator=g)).to(dtype).cuda()


def inside(t, start, gap, fill):
    """A view with t's values in a larger matrix of `fill`; a row of that before and after."""
    big = torch.full((t.shape[0] + 2, t.shape[1] + start + gap), fill, dtype=t.dtype, device="cuda")
    v = big[1:-1, start:start + t.shape[1]]
    v.copy_(t)
    return big, v


def room(rows, width, dtype, start, gap):
    return inside(torch.full((rows, width), 33, dtype=dtype, device="cuda"), start, gap, 33)


def kept(big, v):
    """The marks around the view are there."""
    rest = big.clone()
    rest[1:-1, v.storage_offset() % big.shape[1]:][:, :v.shape[1]] = 33
    return bool((rest == 33).all())


def ends_in_nan(w):
    return torch.cat([w, torch.full((32,), float("nan"), dtype=w.dtype, device="cuda")])[:w.numel()]


@pytest.mark.parametrize("start,gap", [(0, 8), (1, 2), (3, 4), (8, 0)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_forward_and_bytes(kr, width, dtype, start, gap):
    print("norm rows", width, dtype, start, gap, flush=True)
    (x, r), w = make(width, dtype, 2)
    want, held = kr.add_rms_norm(x, w, r), kr.add_rms_norm_bytes(x, w, r)
    (_, xv), (_, rv) = (inside(t, start, gap, float("nan")) for t in (x, r))
    w2 = ends_in_nan(w)
    outs = [room(ROWS, width, dtype, start, gap + 5), room(ROWS, width, dtype, start + 2, gap + 1)]
    f = torch.full((ROWS + 2,), 33.0, device="cuda")
    ld = width + start + gap
    (sb, sv), (ob, ov) = outs
    kr._check("norm", kr._lib.kr_add_rms_norm(
        CODE[dtype], ROWS, width, kr._ptr(xv), ld, kr._ptr(rv), ld, kr._ptr(w2), 1e-6, kr._ptr(sv),
        sb.shape[1], kr._ptr(ov), ob.shape[1], kr._ptr(f[1:]), kr._stream()))
    assert torch.equal(sv, want.sum) and torch.equal(ov, want.out)
    assert torch.equal(f[1:-1], want.rstd) and f[0] == 33 and f[-1] == 33
    assert kept(sb, sv) and kept(ob, ov)

    qb, qv = room(ROWS, width, torch.int8, start, gap + 3)
    sb, sv = room(ROWS, width, dtype, start, gap + 5)
    scale = torch.full((ROWS + 2,), 33.0, device="cuda")
    kr._check("bytes", kr._lib.kr_add_rms_norm_bytes(
        CODE[dtype], ROWS, width, kr._ptr(xv), ld, kr._ptr(rv), ld, kr._ptr(w2), 1e-6, kr._ptr(sv),
        sb.shape[1], kr._ptr(qv), qb.shape[1], kr._ptr(scale[1:]), None, kr._stream()))
    assert torch.equal(qv, held.q) and torch.equal(sv, held.sum)
    assert torch.equal(scale[1:-1], held.scale) and scale[0] == 33 and scale[-1] == 33
    assert kept(qb, qv) and kept(sb, sv)
    # and as the binding takes views
    again = kr.add_rms_norm(xv, w2, rv)
    assert torch.equal(again.out, want.out) and torch.equal(again.sum, want.sum)


@pytest.mark.parametrize("start,gap", [(0, 8), (1, 2), (3, 4), (8, 0)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_backward(kr, width, dtype, start, gap):
    print("norm back rows", width, dtype, start, gap, flush=True)
    (s, g, d), w = make(width, dtype, 3)
    f = (1 / s.float().square().mean(-1).sqrt())
    want, dw = kr.add_rms_norm_backward(g, s, w, f, d)
    (_, sv), (_, gv), (_, dv) = (inside(t, start, gap, float("nan")) for t in (s, g, d))
    w2 = ends_in_nan(w)
    xb, xv = room(ROWS, width, dtype, start + 1, gap + 3)
    got = torch.full((width + 2,), 33.0, device="cuda")
    ld = width + start + gap
    wsb = kr._lib.kr_add_rms_norm_backward_workspace(CODE[dtype], ROWS, width)
    ws = torch.full((wsb + 64,), 255, dtype=torch.uint8, device="cuda")  # NaN wherever it is read
    kr._check("back", kr._lib.kr_add_rms_norm_backward(
        CODE[dtype], ROWS, width, kr._ptr(gv), ld, kr._ptr(sv), ld, kr._ptr(w2), kr._ptr(f),
        kr._ptr(dv), ld, kr._ptr(xv), xb.shape[1], kr._ptr(got[1:]), kr._ptr(ws), wsb,
        kr._stream()))
    assert torch.equal(xv, want) and torch.equal(got[1:-1], dw)
    assert kept(xb, xv) and got[0] == 33 and got[-1] == 33 and (ws[wsb:] == 255).all()
    again = kr.add_rms_norm_backward(gv, sv, w2, f, dv)
    assert torch.equal(again[0], want) and torch.equal(again[1], dw)
