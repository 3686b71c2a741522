"""Products of held values, every byte at every scale: each output is one product of two values, so that
nothing is added to hide what a value became.

Tolerances.  None from 2^-126 on: a product of two e4m3 values has 8 significant bits and is exact in
bfloat16 and in 32 bits, whatever the scales.  Where a value or the result is below 2^-126 the result may be
0.  If it is not, a value below was rounded to bfloat16's step there, 2^-133, and is off by 2^-134 times the other
value, and a result below is rounded to its type's step: 2^-134 again, or 2^-150 in 32 bits.  (Both values
below: the result is far under 2^-134.)"""

import pytest
import torch

from tests.scaled_form import in_order

pytestmark = pytest.mark.gpu

LEAST, MOST = 2.0 ** -126, 2.0 ** 128
# few rows; tiles of 128 x 128 and 128 x 64, with split sums; tiles of 256 x 256
SHAPES = [(1, 254, 254), (16, 254, 254), (40, 254, 254), (300, 254, 254), (4096, 4096, 4)]
# (scale bytes of a, of b)
SCALES = {"every a": ((0, 254), (125, 129)), "every b": ((125, 129), (0, 254)),
          "low a, high b": ((0, 60), (194, 254)), "high a, low b": ((194, 254), (0, 60)),
          "a of 0": ((0, 0), (100, 160)), "b of 0": ((100, 160), (0, 0))}


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def held(rows, blocks, scales, seed):
    """(values of e4m3, scale bytes) [rows][blocks * 128]: all finite bytes, and all bytes of `scales` in turn;
    0 where the value would be past 32 bits."""
    g = torch.Generator().manual_seed(seed)
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    every = every[torch.isfinite(every)]
    q = every[torch.randint(0, len(every), (rows, blocks, 128), generator=g)].double()
    lo, hi = scales
    # along a row and along the diagonal in steps of 7 and 8: through all of 255, 61 or 5
    byte = lo + (torch.arange(rows)[:, None] + 7 * torch.arange(blocks) + seed) % (hi - lo + 1)
    unit = torch.ldexp(torch.ones(byte.shape, dtype=torch.float64), byte - 127)[:, :, None]
    return torch.where((q * unit).abs() < MOST, q, 0.0), byte, unit


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,blocks", SHAPES)
@pytest.mark.parametrize("which", SCALES)
def test_every_byte_at_every_scale(kr, which, m, n, blocks, dtype):
    """Row j of b has one value, in block j: output (i, j) is its product with one value of a."""
    a, ea, ua = held(m, blocks, SCALES[which][0], 1)
    b, eb, ub = held(n, blocks, SCALES[which][1], 2)
    j = torch.arange(n)
    block, place = j % blocks, j * 37 % 128
    one = torch.zeros_like(b)
    one[j, block, place] = b[j, block, place]
    va, vb = (a * ua)[:, block, place], (b * ub)[j, block, place]
    got = kr.scaled_matmul(
        kr.Scaled(a.reshape(m, -1).to(torch.float8_e4m3fn).cuda(), in_order(ea).cuda()),
        kr.Scaled(one.reshape(n, -1).to(torch.float8_e4m3fn).cuda(), in_order(eb).cuda()), dtype)
    got, want = got.double().cpu(), va * vb
    there = want.abs() < MOST  # in 32 bits
    must = (va.abs() >= LEAST) & (vb.abs() >= LEAST) & (want.abs() >= LEAST)
    none = torch.zeros_like(want)
    step = 2.0 ** -134
    off = step * (torch.where(va.abs() < LEAST, vb.abs().expand_as(va), none) +
                  torch.where(vb.abs() < LEAST, va.abs(), none) + torch.where(want.abs() < LEAST, 1.0, none))
    right = (got == want) | (~must & ((got == 0) | ((got - want).abs() <= off)))
    bad = there & ~right
    assert not bad.any(), "%d of %d, the first at a %g * 2^%d, b %g * 2^%d: %g" % (
        int(bad.sum()), int((there & must).sum()),
        *[f(*bad.nonzero()[0].tolist()) for f in (
            lambda x, y: a[x, block[y], place[y]], lambda x, y: ea[x, block[y]] - 127,
            lambda x, y: b[y, block[y], place[y]], lambda x, y: eb[y, block[y]] - 127,
            lambda x, y: got[x, y])])
    seen = there & must
    assert seen.sum() > 0.3 * m * n
    if which == "every a":  # the scales of no held value are left out
        assert len(ea[:, block][seen].unique()) >= 240
    if which == "every b":
        assert len(eb[j, block][seen.any(0)].unique()) >= 240


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(1, 40, 700), (16, 40, 700), (100, 300, 700), (4096, 4096, 300)])
def test_what_is_no_number(kr, m, n, k, dtype):
    """The byte of a NaN and the scale of a NaN, beside any value, a 0 or a value at the other operand's end: NaN
    through the whole row or column, and nowhere else."""
    g = torch.Generator().manual_seed(3)
    blocks = -(-k // 128)
    a, b = (torch.randint(0, 0x7F, (r, k), generator=g, dtype=torch.uint8) for r in (m, n))
    ea, eb = (torch.randint(110, 130, (r, blocks), generator=g) for r in (m, n))
    a[:, 5], b[:, 6] = 0, 0
    good = [t.clone() for t in (a, ea, b, eb)]
    bad = torch.zeros(m, n, dtype=torch.bool)
    a[m // 2, k - 1] = 0xFF
    bad[m // 2] = True
    b[3, 5], b[n - 1, 7] = 0x7F, 0xFF  # against zeros, too
    eb[7, 1], eb[8, blocks - 1] = 255, 255
    bad[:, [3, 7, 8, n - 1]] = True
    if m > 1:
        ea[m - 1, 0] = 255
        bad[m - 1] = True

    def product(a, ea, b, eb):
        return kr.scaled_matmul(kr.Scaled(a.view(torch.float8_e4m3fn).cuda(), in_order(ea).cuda()),
                                kr.Scaled(b.view(torch.float8_e4m3fn).cuda(), in_order(eb).cuda()), dtype).cpu()

    got, want = product(a, ea, b, eb), product(*good)
    assert torch.equal(got.isnan(), bad) and not want.isnan().any()
    assert torch.equal(got[~bad], want[~bad])
    for q, e in ((a, ea), (b, eb)):
        v = kr.scaled_values(kr.Scaled(q.view(torch.float8_e4m3fn).cuda(), in_order(e).cuda()), dtype).cpu()
        no = (q & 0x7F == 0x7F) | (e == 255).repeat_interleave(128, 1)[:, :k]
        assert torch.equal(v.isnan(), no)
