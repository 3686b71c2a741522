"""Matrices whose offsets pass 32 bits: more than 2^31 elements or 4 GiB.  The rows at either end
are checked against the operator on those rows alone (each row stands for itself; a sum over
rows is checked by giving most rows nothing to add)."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


@pytest.fixture(autouse=True)
def freed():
    yield
    torch.cuda.empty_cache()


def normal(*shape, seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty(shape, dtype=dtype, device="cuda")
    for part in x.split(1 << 16):  # no 32-bit copy of the whole
        part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    return x


def ends(n):
    return (slice(0, 40), slice(n - 40, n))


def test_norm(kr):
    rows, width = 530000, 4096  # 2.17e9 elements
    x, r, w = normal(rows, width), normal(rows, width, seed=1), normal(width, seed=2)
    full = kr.add_rms_norm(x, w, r)
    held = kr.add_rms_norm_bytes(x, w, r)
    for e in ends(rows):
        some, few = kr.add_rms_norm(x[e], w, r[e]), kr.add_rms_norm_bytes(x[e], w, r[e])
        assert torch.equal(full.out[e], some.out) and torch.equal(full.sum[e], some.sum)
        assert torch.equal(held.q[e], few.q) and torch.equal(held.scale[e], few.scale)
    del held, r
    dx, _ = kr.add_rms_norm_backward(full.out, x, w, full.rstd)
    for e in ends(rows):
        some, _ = kr.add_rms_norm_backward(full.out[e], x[e], w, full.rstd[e])
        assert torch.equal(dx[e], some)


def test_narrow_rows_of_several_launches(kr):
    rows, width = (1 << 21) + 1000, 24  # more rows than one launch takes
    x, w = normal(rows, width), normal(width, seed=2)
    full = kr.add_rms_norm(x, w)
    for e in ends(rows) + (slice((1 << 21) - 20, (1 << 21) + 20),):
        some = kr.add_rms_norm(x[e], w)
        assert torch.equal(full.out[e], some.out) and torch.equal(full.rstd[e], some.rstd)


def test_bytes_many_tokens_and_many_channels(kr):
    big, k = 1100000, 4096  # 4.5e9 bytes
    a = torch.empty(big, k, dtype=torch.int8, device="cuda")
    for i, part in enumerate(a.split(1 << 18)):
        part.random_(-127, 128, generator=torch.Generator(device="cuda").manual_seed(i))
    b = a[5000:5048].clone()
    sa, sb = torch.rand(big, device="cuda"), torch.rand(48, device="cuda")
    full = kr.byte_matmul(a, sa, b, sb)
    wide = kr.byte_matmul(b, sb, a, sa)
    few = kr.byte_matmul(b[:3], sb[:3], a, sa)
    for e in ends(big):
        exact = (a[e].double() @ b.double().t()).float()
        assert torch.equal(full[e], (exact * sa[e][:, None] * sb).bfloat16())
        assert torch.equal(wide[:, e], (exact.t() * sb[:, None] * sa[e]).bfloat16())
        assert torch.equal(few[:, e], (exact.t()[:3] * sb[:3, None] * sa[e]).bfloat16())


def test_gated_forward_and_backward(kr):
    rows, width, hidden = 140000, 64, 16384  # outputs of 4.6 GB, dg and du of 9.2 GB
    x = normal(rows, width)
    wg, wu = normal(hidden, width, seed=1) / 8, normal(hidden, width, seed=2) / 8
    h = kr.gated_projection(x, wg, wu)
    for e in ends(rows):
        assert torch.equal(h[e], kr.gated_projection(x[e], wg, wu))
    # only the last 40 rows have a gradient: the weights' sums are theirs
    dh = h.zero_()
    last = slice(rows - 40, rows)
    dh[last] = normal(40, hidden, seed=3)
    dx, dwg, dwu = kr.gated_projection_backward(dh, x, wg, wu)
    assert (dx[:rows - 40] == 0).all()
    x64, g64, u64, d64 = x[last].double(), wg.double(), wu.double(), dh[last].double()
    g, u = x64 @ g64.t(), x64 @ u64.t()
    p = torch.sigmoid(g)
    dg, du = d64 * u * (p + g * p * (1 - p)), d64 * g * p
    # three roundings to bfloat16 (dg or du, the sum, and the sums' own errors well below), each
    # relative to the sizes of what is added up
    for got, want, size in ((dx[last], dg @ g64 + du @ u64, dg.abs() @ g64.abs() + du.abs() @ u64.abs()),
                            (dwg, dg.t() @ x64, dg.abs().t() @ x64.abs()),
                            (dwu, du.t() @ x64, du.abs().t() @ x64.abs())):
        assert ((got.double() - want).abs() <= 3 * 2.0 ** -8 * size).all()
