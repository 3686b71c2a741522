"""The norm's weight gradient over many rows: what a slot adds in turn in 32 bits."""

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


@pytest.fixture(autouse=True)
def freed():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", [(530001, 24), (100003, 1000), (40001, 4096), (3000, 9001),
                                        (20011, 16390)])
def test_weight_gradient_of_many_rows(kr, rows, width, dtype):
    """A column's sum in 32 bits against 64.  A slot adds at most rows / slots terms in turn (256
    slots or more, 64 where rows are read again), the slots at most 32 runs of 64: (rows / slots +
    100) 2^-24 relative to the terms' sizes."""
    g = torch.Generator(device="cuda").manual_seed(rows)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)

    s, dout, w = normal(rows, width), normal(rows, width), normal(width)
    f = torch.rsqrt(s.float().square().mean(-1) + 1e-6)
    _, dw = kr.add_rms_norm_backward(dout, s, w, f)
    want, size = (torch.zeros(width, dtype=torch.float64, device="cuda") for _ in range(2))
    for i in range(0, rows, 4096):  # no 64-bit copy of the whole
        p = slice(i, i + 4096)
        t = dout[p].double() * s[p].double() * f[p].double()[:, None]
        want += t.sum(0)
        size += t.abs().sum(0)
    run = rows / (64 if width > 16384 else 256)
    assert ((dw.double() - want).abs() <= (run + 100) * 2.0 ** -24 * size).all()
