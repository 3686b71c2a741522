"""Product of 8-bit integers with scales against exact integer sums.  The sum is exact, the
scales are applied as (sum * sa) * sb in 32 bits and the result is rounded once, so every output
has to match bit for bit."""

import pytest
import torch

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 1), (1, 8, 16), (1, 1000, 4096), (2, 3, 5), (3, 64, 2059), (15, 33, 128),
          (16, 129, 100), (17, 40, 77), (33, 300, 1024), (64, 512, 64), (100, 130, 16),
          (128, 128, 128), (129, 257, 520), (333, 501, 259), (1000, 16, 48), (4096, 4100, 144)]


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def make(m, n, k, seed):
    g = torch.Generator().manual_seed(seed)
    a = torch.randint(-128, 128, (m, k), generator=g, dtype=torch.int8).cuda()
    b = torch.randint(-128, 128, (n, k), generator=g, dtype=torch.int8).cuda()
    sa = torch.exp(torch.randn(m, generator=g)).cuda()
    sb = torch.exp(torch.randn(n, generator=g)).cuda()
    return a, sa, b, sb


def want(a, sa, b, sb, dtype):
    s = a.double() @ b.double().t()  # exact: below 2^53
    return ((s.float() * sa[:, None]) * sb[None, :]).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES)
def test_product(kr, shape, dtype):
    print("bytes", shape, dtype, flush=True)
    a, sa, b, sb = make(*shape, sum(shape))
    sa = sa / shape[2]
    got = kr.byte_matmul(a, sa, b, sb, dtype=dtype)
    assert torch.equal(got, want(a, sa, b, sb, dtype))


@pytest.mark.parametrize("m", [1, 20, 300])
def test_largest_sums(kr, m):
    """The longest row at the lowest values: the sum is 2^14 * 131071, just below 2^31; and one
    with alternating signs that ends near 0."""
    k = 131071
    a = torch.full((m, k), -128, dtype=torch.int8, device="cuda")
    b = torch.full((9, k), -128, dtype=torch.int8, device="cuda")
    b[1::2, ::2] = 127
    one = torch.ones(m, device="cuda")
    got = kr.byte_matmul(a, one, b, torch.ones(9, device="cuda"), dtype=torch.float32)
    assert torch.equal(got, want(a, one, b, torch.ones(9, device="cuda"), torch.float32))
    assert float(got[0, 0]) == 2.0 ** 14 * k


@pytest.mark.parametrize("gap,start", [(16, 16), (3, 0), (7, 5)])
def test_strides(kr, gap, start):
    a, sa, b, sb = make(70, 90, 208, 3)

    def inside(t):
        big = torch.full((t.shape[0] + 2, t.shape[1] + start + gap), 77, dtype=torch.int8,
                         device="cuda")
        v = big[1:-1, start:start + t.shape[1]]
        v.copy_(t)
        return v

    assert torch.equal(kr.byte_matmul(a, sa, b, sb), kr.byte_matmul(inside(a), sa, inside(b), sb))
    c = kr.byte_matmul(a.reshape(2, 35, 208), sa.reshape(2, 35), b, sb)
    assert c.shape == (2, 35, 90)
    assert torch.equal(kr.byte_matmul(a, sa, b.t().contiguous().t(), sb),
                       kr.byte_matmul(a, sa, b, sb))


def test_scales_that_are_not_finite(kr):
    a, sa, b, sb = make(40, 50, 64, 5)
    clean = kr.byte_matmul(a, sa, b, sb)
    sa[7] = float("nan")
    sb[3] = 0.0
    got = kr.byte_matmul(a, sa, b, sb)
    keep = torch.arange(40) != 7
    assert got[7].isnan().all() and (got[keep][:, 3] == 0).all()
    cols = torch.arange(50) != 3
    assert torch.equal(got[keep][:, cols], clean[keep][:, cols])


def test_no_rows(kr):
    a, sa, b, sb = make(1, 12, 32, 1)
    assert kr.byte_matmul(a[:0], sa[:0], b, sb).shape == (0, 12)


def test_from_the_norm(kr):
    """Norm in 8 bits and the product, as a projection uses them: within the held values' half
    steps of the product of the norm itself."""
    g = torch.Generator().manual_seed(2)
    x = torch.randn(50, 320, generator=g).cuda()
    w = torch.ones(320).cuda()
    n = kr.add_rms_norm_bytes(x, w)
    _, _, b, sb = make(1, 64, 320, 4)
    got = kr.byte_matmul(n.q, n.scale, b, sb, dtype=torch.float32)
    full = kr.add_rms_norm(x, w).out.double() @ (b.double() * sb.double()[:, None]).t()
    off = 0.5001 * n.scale.double()[:, None] * (b.double().abs() * sb.double()[:, None]).sum(1)
    assert ((got.double() - full).abs() <= off + 1e-5 * full.abs()).all()
