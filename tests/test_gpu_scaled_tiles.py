"""The 8-bit product on its large tiles and with split sums, at odd sizes and odd numbers of steps (the
shapes of the 8-bit integers' tiles, whose cut is pinned on the CPU; outputs of 32 bits take small tiles
there): whole numbers, exactly, and every place of a tile by rows and columns that differ."""

import pytest
import torch

from tests.block_shapes import BYTES
from tests.scaled_form import in_order, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def parts(rows, k, seed, most):
    g = torch.Generator().manual_seed(seed)
    v = torch.randint(-most, most + 1, (rows, k), generator=g).double()
    e = torch.randint(-1, 2, (rows, -(-k // 128)), generator=g) + 127
    return v, e


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", sorted(BYTES) + [(300, 700, 128), (513, 1024, 127), (2100, 2100, 384)])
def test_whole_numbers(kr, shape, dtype):
    """Sums of whole numbers to 4 at scales from 1/2 to 2: 16 * 4 * 14401 < 2^20 in units of 1/4, exact in 32
    bits, and a block's products within 2^4 of each other; rounded once."""
    m, n, k = shape
    a, ea = parts(m, k, 1, 4)
    b, eb = parts(n, k, 2, 4)
    a[:, ::37] = 0  # holes
    got = kr.scaled_matmul(kr.Scaled(a.to(torch.float8_e4m3fn).cuda(), in_order(ea).cuda()),
                           kr.Scaled(b.to(torch.float8_e4m3fn).cuda(), in_order(eb).cuda()), dtype)
    want = (values(a, ea).cuda() @ values(b, eb).cuda().t()).to(dtype)
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,width,hidden", [
    (4917, 5056, 832), (2048, 2304, 4352), (1000, 2000, 1500), (16, 4100, 600), (17, 300, 5000), (100, 130, 16000),
    (9000, 140, 150), (300, 6000, 700), (1, 512, 640)])
def test_linear_gradients(kr, rows, width, hidden, dtype):
    """Both gradients' products, alone and in one launch, in tiles of either size, whole and split sums: whole
    numbers to 4 are held as they are, their sums (16 * 16000 < 2^18) are exact in 32 bits, a block's products
    within 2^4 of each other."""
    g = torch.Generator().manual_seed(rows)
    x, w, d = (torch.randint(-4, 5, s, generator=g).to(dtype).cuda()
               for s in ((rows, width), (hidden, width), (rows, hidden)))
    size = 0.0625 if dtype == torch.float16 else 1.0  # sums of float16 stay below 65,504
    y = kr.scaled_linear(x, w * size)
    assert torch.equal(y, (x.double() @ w.double().t() * size).to(dtype))
    want = ((d.double() @ w.double() * size).to(dtype), (d.double().t() @ x.double() * size).to(dtype))
    both = kr.scaled_linear_backward(d * size, x, w)
    one, none = kr.scaled_linear_backward(d * size, x, w, need=(True, False))
    assert none is None
    none, two = kr.scaled_linear_backward(d * size, x, w, need=(False, True))
    assert none is None
    for a, b in zip((*both, one, two), (*want, *want)):
        assert torch.equal(a, b)


def test_same_bits_again(kr):
    """Twice, and on another stream at the same time: the same bits (no order changes)."""
    g = torch.Generator().manual_seed(3)
    for m, n, k in ((700, 6000, 14401), (333, 501, 8200), (40, 5001, 2059)):
        a = kr.scaled_hold(torch.randn(m, k, generator=g).cuda()).plain
        b = kr.scaled_hold(torch.randn(n, k, generator=g).cuda()).plain
        side = torch.cuda.Stream()
        for dtype in (torch.bfloat16, torch.float32):
            one = kr.scaled_matmul(a, b, dtype)
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                two = kr.scaled_matmul(a, b, dtype)
            three = kr.scaled_matmul(a, b, dtype)
            torch.cuda.synchronize()
            assert torch.equal(one, two) and torch.equal(one, three)


def test_past_32_bit_offsets(kr):
    """Operands and outputs of more than 2^32 bytes, checked in their last rows."""
    m, n, k = 280000, 8200, 16000
    g = torch.Generator().manual_seed(4)
    part = torch.randint(-4, 5, (280, k), generator=g).to(torch.float8_e4m3fn).cuda()
    bv = torch.randint(-4, 5, (n, k), generator=g).to(torch.float8_e4m3fn).cuda()
    av = part.view(torch.uint8).repeat(1000, 1).view(torch.float8_e4m3fn)
    unit = torch.full((125, 280064), 127, dtype=torch.uint8, device="cuda")
    got = kr.scaled_matmul(kr.Scaled(av, unit), kr.Scaled(bv, unit[:, :8320]), torch.bfloat16)
    want = (part.float().double() @ bv.float().double().t()).bfloat16()
    for r in (0, 137 * 280, 500 * 280, 999 * 280):
        assert torch.equal(got[r:r + 280], want), r
