"""Values held in 8-bit floating point: every byte and every scale against the definition (holding is one
rounding, so that they are equal), both forms, at sizes around the 128 of a block, with rows apart,
blocks of zeros, of the smallest and largest magnitudes, and of what is no number."""

import pytest
import torch

from tests.scaled_form import hold, in_order, values

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
SHAPES = [(1, 1), (1, 128), (1, 4096), (3, 7), (5, 129), (127, 15), (128, 128), (129, 200), (16, 513),
          (300, 1000), (513, 300), (1031, 96), (2, 5000), (5000, 2)]


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def make(rows, width, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, width, generator=g) * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=g))
    return x.to(dtype)


def check(got, x, square, kr):
    q, byte = hold(x, square)
    assert got.q.shape == x.shape and got.q.dtype == torch.float8_e4m3fn
    assert torch.equal(got.q.float().cpu().double(), q)
    assert torch.equal(got.scale.cpu(), in_order(byte))
    for dtype in TYPES:
        back = kr.scaled_values(got, dtype).cpu()
        assert torch.equal(back.nan_to_num(-7.0), values(q, byte).to(dtype).nan_to_num(-7.0))


@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", SHAPES)
def test_forms(kr, rows, width, dtype, square):
    x = make(rows, width, dtype, rows + width)
    both = kr.scaled_hold(x.cuda(), square, crossed=True)
    check(both.plain, x, square, kr)
    check(both.crossed, x.t(), square, kr)
    one, two = kr.scaled_hold(x.cuda(), square), kr.scaled_hold(x.cuda(), square, False, True)
    assert one.crossed is None and two.plain is None
    for a, b in ((one.plain, both.plain), (two.crossed, both.crossed)):
        assert torch.equal(a.q.view(torch.uint8), b.q.view(torch.uint8))
        assert torch.equal(a.scale, b.scale)
        # the room behind the rows is zeros
        store = a.q.as_strided((a.q.shape[0], a.room), (a.room, 1)).view(torch.uint8)
        assert not store[:, a.q.shape[1]:].any()


@pytest.mark.parametrize("square", [False, True])
def test_extremes(kr, square):
    """Blocks of zeros, of subnormal, largest and bordering magnitudes, of NaN and infinities."""
    rows = []
    for v in (0.0, 2.0 ** -149, 2.0 ** -130, 2.0 ** -127, 2.0 ** -119, 2.0 ** -118, 3.4e38, 448.0,
              448.0 + 2.0 ** -15, -447.99, 1.75, 1.7500001, 2.0 ** -9, float("nan"), float("inf"),
              float("-inf")):
        row = torch.linspace(-1, 1, 300) * (v if abs(v) < 1e300 else 1.0)
        row[200] = v
        rows.append(row)
    x = torch.stack(rows)
    x = x.repeat_interleave(128, 0) if square else x
    both = kr.scaled_hold(x.cuda(), square, crossed=True)
    check(both.plain, x, square, kr)
    check(both.crossed, x.t(), square, kr)
    h = x.half()  # with its infinities and subnormals
    check(kr.scaled_hold(h.cuda(), square).plain, h, square, kr)


def test_ties(kr):
    """Halves between neighbours go to the even one."""
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    every = every[torch.isfinite(every)].sort().values
    x = torch.full((2, 256), 448.0)
    half = (every[1:] + every[:-1]) / 2
    x[0, :127], x[1, :126] = half[:127], half[127:253]
    check(kr.scaled_hold(x.cuda()).plain, x, False, kr)


@pytest.mark.parametrize("dtype", TYPES)
def test_strides(kr, dtype):
    store = make(140, 333, dtype, 4).cuda()
    for x in (store[:, 1:302], store[:, 5:], store.t(), store[::2, 3:], store[:1].expand(50, 333),
              store[:, :330].reshape(7, 20, 330)):
        both = kr.scaled_hold(x, crossed=True)
        flat = x.reshape(-1, x.shape[-1]).cpu()
        q, byte = hold(flat)
        assert both.plain.q.shape == x.shape
        assert torch.equal(both.plain.q.reshape(flat.shape).float().cpu().double(), q)
        assert torch.equal(both.plain.scale.cpu(), in_order(byte))
        assert kr.scaled_values(both.plain).shape == x.shape
        check(both.crossed, flat.t(), False, kr)


def test_rows_apart_keep_their_gaps(kr):
    """The C call on outputs that are parts of larger ones: what lies past a row's room stays."""
    import ctypes

    x = make(130, 300, torch.float32, 6).cuda()
    q = torch.full((131, 350), 9, dtype=torch.uint8, device="cuda")
    qt = torch.full((301, 150), 9, dtype=torch.uint8, device="cuda")
    s = torch.full((4, 300), 9, dtype=torch.uint8, device="cuda")
    st = torch.full((3, 400), 9, dtype=torch.uint8, device="cuda")
    plain = kr.KrScaled(q.data_ptr() + 3, 350, 301, s.data_ptr(), 300)
    crossed = kr.KrScaled(qt.data_ptr(), 150, 130, st.data_ptr(), 400)
    assert kr._lib.kr_scaled_hold(0, 130, 300, x.data_ptr(), 300, 0, ctypes.byref(plain),
                                  ctypes.byref(crossed), kr._raw_stream(0)) == kr.KR_OK
    want = kr.scaled_hold(x, crossed=True)
    flat = q.view(-1)[3:3 + 130 * 350].view(130, 350)
    assert torch.equal(flat[:, :300], want.plain.q.view(torch.uint8)) and not flat[:, 300].any()
    assert (flat[:, 301:347] == 9).all() and (q[130, 3:] == 9).all()
    assert torch.equal(qt[:300, :130], want.crossed.q.view(torch.uint8))
    assert (qt[:, 130:] == 9).all() and (qt[300] == 9).all()
    assert torch.equal(s[:3, :256], want.plain.scale) and (s[:, 256:] == 9).all() and (s[3] == 9).all()
    assert torch.equal(st[:2, :384], want.crossed.scale) and (st[2] == 9).all()


def test_empty(kr):
    x = torch.zeros(0, 300).cuda()
    both = kr.scaled_hold(x, crossed=True)
    assert both.plain.q.shape == (0, 300) and both.crossed.q.shape == (300, 0)
    assert kr.scaled_values(both.plain).shape == (0, 300)


def test_large(kr):
    """Past 32-bit offsets: 300,000 rows of 16,000, checked at their ends; a pattern that repeats."""
    rows, width = 300000, 16000
    part = make(128, width, torch.bfloat16, 7).cuda()
    x = part.repeat(-(-rows // 128), 1)[:rows]
    both = kr.scaled_hold(x, crossed=True)
    del x
    want = kr.scaled_hold(part, crossed=True)
    for r in (0, 134144, rows // 128 * 128 - 128):
        assert torch.equal(both.plain.q[r:r + 128].view(torch.uint8),
                           want.plain.q.view(torch.uint8)), r
        assert torch.equal(both.plain.scale[:, r:r + 128], want.plain.scale)
        assert torch.equal(both.crossed.q[:, r:r + 128].view(torch.uint8),
                           want.crossed.q.view(torch.uint8))
        assert torch.equal(both.crossed.scale[r // 128], want.crossed.scale[0])
    del both.crossed.q
    back = kr.scaled_values(both.plain, torch.bfloat16)
    assert torch.equal(back[rows // 128 * 128 - 128:rows // 128 * 128],
                       kr.scaled_values(want.plain, torch.bfloat16))


@pytest.mark.parametrize("square", [False, True])
def test_past_32_bit_offsets(kr, square):
    """More than 2^32 values, one pattern of 128 rows over and over, strided: each form is the pattern's over
    and over, and so are the values that it holds."""
    width, n = 8200, 4097
    part = make(128, width, torch.bfloat16, 6).cuda()
    x = torch.empty(n * 128, width + 3, dtype=torch.bfloat16, device="cuda")[:, 1:-2]
    x.copy_(part.repeat(n, 1))
    one = kr.scaled_hold(part, square, crossed=True)
    many = kr.scaled_hold(x, square, crossed=True)
    del x
    for k in range(0, n, 241):
        rows = slice(k * 128, k * 128 + 128)
        assert torch.equal(many.plain.q[rows].view(torch.uint8), one.plain.q.view(torch.uint8)), k
        assert torch.equal(many.crossed.q[:, rows].view(torch.uint8), one.crossed.q.view(torch.uint8)), k
        assert torch.equal(many.plain.scale[:, rows], one.plain.scale[:, :128]), k
        assert torch.equal(many.crossed.scale[k], one.crossed.scale[0]), k
    rows = slice((n - 1) * 128, n * 128)
    assert torch.equal(many.plain.q[rows].view(torch.uint8), one.plain.q.view(torch.uint8))
    assert torch.equal(many.crossed.q[:, rows].view(torch.uint8), one.crossed.q.view(torch.uint8))
    assert torch.equal(many.crossed.scale[n - 1], one.crossed.scale[0])
    small = kr.scaled_values(one.plain, torch.bfloat16)
    back = kr.scaled_values(many.plain, torch.bfloat16)
    for k in (0, n // 2, n - 1):
        assert torch.equal(back[k * 128:k * 128 + 128], small), k
