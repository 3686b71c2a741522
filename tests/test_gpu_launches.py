"""Rows past one launch: dropout and the values of a held matrix go on where the launch before ended, at
either side of its edge (tests/dealt.py says where that is)."""

import pytest
import torch

from tests.dealt import rows_a_launch
from tests.philox import factor
from tests.scaled_form import hold, in_order, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def places(edge, rows, n):
    """First rows of runs of n: at the beginning, before, across and after the edge, at the end."""
    return sorted({0, edge // 2, edge - n, edge - n // 2, edge, rows - n})


@pytest.mark.parametrize("width,residual", [(1, True), (17, False), (2048, False)])
def test_dropout(kr, width, residual):
    """Kept values are whole numbers times 2: exact."""
    edge = rows_a_launch(-(-width // 8))
    rows, n = edge + 40, 16
    # a row's values from its number: a row taken for another shows
    part = torch.arange(1, 252, dtype=torch.bfloat16, device="cuda")[:, None].expand(251, width)
    x = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda")
    whole = rows // 251 * 251
    x[:whole].view(-1, 251, width).copy_(part.expand(whole // 251, 251, width))
    x[whole:] = part[:rows - whole]
    r = None
    if residual:
        r = torch.empty_like(x)
        r[:rows // 2] = 3
        r[rows // 2:] = 5
    got = kr.dropout(x, 0.5, 11, 5, r)
    for row0 in places(edge, rows, n):
        f = factor(n, width, 0.5, 11, 5, row0)
        want = x[row0:row0 + n].double().cpu() * f
        if residual:
            want = want + r[row0:row0 + n].double().cpu()
        assert torch.equal(got[row0:row0 + n].double().cpu(), want.bfloat16().double()), row0


def test_values_of_many_rows(kr):
    """Narrow rows, 2^29 a launch: 253 rows of different scales over and over."""
    width = 9
    edge = rows_a_launch(-(-width // 4))
    rows, n = edge + 300, 140
    g = torch.Generator().manual_seed(1)
    x = torch.randn(253, width, generator=g) * torch.exp2(torch.randint(-20, 20, (253, 1), generator=g))
    q, byte = hold(x)
    many = -(-rows // 253)
    held = q.to(torch.float8_e4m3fn).view(torch.uint8).cuda().repeat(many, 1)[:rows]
    flat = torch.zeros(-(-rows // 128) * 128, dtype=torch.uint8, device="cuda")
    flat[:rows] = byte[:, 0].to(torch.uint8).cuda().repeat(many)[:rows]
    scale = flat.view(-1, 8, 16).transpose(1, 2).reshape(1, -1)
    del flat
    assert torch.equal(scale[:, :128].cpu(), in_order(byte[:128]))
    got = kr.scaled_values(kr.Scaled(held.view(torch.float8_e4m3fn), scale), torch.float32)
    want = values(q, byte)
    for row0 in places(edge, rows, n):
        assert torch.equal(got[row0:row0 + n].double().cpu(), want[torch.arange(row0, row0 + n) % 253]), row0


@pytest.mark.parametrize("rows,width", [(130, (1 << 26) + 261), (128, 1 << 27)])
def test_values_of_wide_rows(kr, rows, width):
    """Rows so wide that fewer than 128, whose scale bytes are neighbours, fill a launch."""
    edge = rows_a_launch(-(-width // 4))
    assert edge < 128
    g = torch.Generator().manual_seed(2)
    every = torch.randint(0, 0x7F, (rows, 1000), generator=g, dtype=torch.uint8)
    byte = torch.randint(80, 160, (rows, 500), generator=g)
    blocks, ld = -(-width // 128), -(-width // 16) * 16
    held = torch.empty(rows, ld, dtype=torch.uint8, device="cuda")
    for i in range(rows):
        held[i] = every[i].cuda().repeat(-(-ld // 1000))[:ld]
    scale = in_order(byte).cuda().repeat(-(-blocks // 500), 1)[:blocks]
    got = kr.scaled_values(kr.Scaled(held[:, :width].view(torch.float8_e4m3fn), scale), torch.float32)
    every = every.view(torch.float8_e4m3fn).double()
    for i in sorted({0, 1, edge - 1, edge, rows - 1}):
        for c0 in (0, width // 2, width - 3000):
            c = torch.arange(c0, c0 + 3000)
            want = every[i, c % 1000] * torch.ldexp(torch.ones(3000, dtype=torch.float64),
                                                    byte[i, c // 128 % 500] - 127)
            assert torch.equal(got[i, c0:c0 + 3000].double().cpu(), want), (i, c0)


@pytest.mark.parametrize("square", [False, True])
def test_hold_of_the_most_rows(kr, square):
    """2^22 squares, the most that is taken, in one launch: three blocks of rows over and over, to the last."""
    rows, width, n = 1 << 29, 3, 384
    g = torch.Generator().manual_seed(3)
    part = (torch.randn(n, width, generator=g) * torch.exp2(torch.randint(-9, 9, (n, 1), generator=g))).bfloat16()
    x = part.cuda().repeat(-(-rows // n), 1)[:rows]
    plain, crossed = hold(part, square), hold(part.t(), square)
    byte, turned = in_order(plain[1]), in_order(crossed[1])
    for forms in (dict(), dict(crossed=True), dict(plain=False, crossed=True)):
        got = kr.scaled_hold(x, square, **forms)
        for block in (0, 1, 1 << 21, (1 << 22) - 2, (1 << 22) - 1):
            i, k = block * 128, block % 3 * 128
            if got.plain is not None:
                assert torch.equal(got.plain.q[i:i + 128].float().cpu().double(), plain[0][k:k + 128]), block
                assert torch.equal(got.plain.scale[:, i:i + 128].cpu(), byte[:, k:k + 128]), block
            if got.crossed is not None:
                assert torch.equal(got.crossed.q[:, i:i + 128].float().cpu().double(),
                                   crossed[0][:, k:k + 128]), block
                assert torch.equal(got.crossed.scale[block].cpu(), turned[block % 3]), block
        del got


def test_layer_norm_gradient_of_long_rows(kr):
    """Rows too long for registers, 2^21 a launch, the gradient over dout: as the first rows alone, and whole
    numbers whose sums over rows are exact below 2^24, so that a row left out or taken twice shows."""
    import ctypes

    rows, width, n, ld = (1 << 21) + 40, 16385, 64, 16392
    t = kr._TYPES[torch.bfloat16]
    g = torch.Generator().manual_seed(4)
    s, d = (torch.randint(-2, 3, (n, width), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    w = torch.ones(width, dtype=torch.bfloat16, device="cuda")
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    few = kr.add_layer_norm_backward(d, s, w, mean[:n], rstd[:n])
    big = [torch.empty(rows, ld, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    whole = rows // n * n
    for b, part in zip(big, (s, d)):
        b[:whole].view(-1, n, ld)[:, :, :width] = part
        b[whole:, :width] = part[:rows - whole]
        b[:, width:] = 7
    times = torch.full((n, 1), float(rows // n), dtype=torch.float64, device="cuda")
    times[:rows - whole] += 1
    want = [(s.double() * d.double() * times).sum(0), (d.double() * times).sum(0)]
    assert max(float((v.abs().double() * times).sum(0).max()) for v in (s.double() * d.double(), d)) < 2 ** 24
    dw, db = torch.empty(width, device="cuda"), torch.empty(width, device="cuda")
    wsb = kr._lib.kr_add_layer_norm_backward_workspace(t, rows, width)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    at = big[1].data_ptr()
    assert kr._lib.kr_add_layer_norm_backward(
        t, rows, width, at, ld, big[0].data_ptr(), ld, w.data_ptr(), mean.data_ptr(), rstd.data_ptr(), None, 0,
        None, at, ld, None, 0, dw.data_ptr(), db.data_ptr(), ws.data_ptr(), wsb, kr._raw_stream(0)) == kr.KR_OK
    edge = 1 << 21
    for row0 in (0, edge - n, edge, rows // n * n - n):
        assert torch.equal(big[1][row0:row0 + n, :width], few[1][:big[1][row0:row0 + n].shape[0]]), row0
        assert (big[1][row0:row0 + n, width:] == 7).all()
    assert torch.equal(dw.double(), want[0]) and torch.equal(db.double(), want[1])
