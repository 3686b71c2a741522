"""The products' large tiles, alone and with split sums, against 64 bits: the tolerances of the
other tests of the same operators (the 8-bit product bit for bit).  That the shapes take such
tiles is pinned in test_block_plans.py."""

import pytest
import torch

from tests import test_gpu_bytes as B
from tests import test_gpu_gated as G
from tests.block_shapes import BYTES, GATED

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


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def inputs(rows, width, hidden, dtype):
    return (normal((rows, width), dtype, 1), normal((hidden, width), dtype, 2, 1.5 / width ** 0.5),
            normal((hidden, width), dtype, 3, 1.0 / width ** 0.5), normal((rows, hidden), dtype, 4))


@pytest.mark.parametrize("dtype,act", [(torch.bfloat16, "silu"), (torch.float16, "gelu")])
@pytest.mark.parametrize("shape", sorted(GATED))
def test_gated(kr, shape, dtype, act):
    print("tiles", shape, dtype, flush=True)
    x, wg, wu, dh = inputs(*shape, dtype)
    w = G.Want(x, wg, wu, dh, act, dtype)
    h = kr.gated_projection(x, wg, wu, act)
    G.near(h, w.h, w.eh, "h")
    got = kr.gated_projection_backward(dh, x, wg, wu, act)
    for g, want, off, what in zip(got, (w.dx, w.dwg, w.dwu), (w.edx, w.edwg, w.edwu),
                                  ("dx", "dwg", "dwu")):
        G.near(g, want, off, what)
    # the same bits again, beside other work
    for _ in range(2):
        assert torch.equal(h, kr.gated_projection(x, wg, wu, act))
        again = kr.gated_projection_backward(dh, x, wg, wu, act)
        assert all(torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", sorted(BYTES))
def test_bytes(kr, shape, dtype):
    print("tiles bytes", shape, dtype, flush=True)
    a, sa, b, sb = B.make(*shape, sum(shape))
    sa = sa / shape[2]
    got = kr.byte_matmul(a, sa, b, sb, dtype=dtype)
    assert torch.equal(got, B.want(a, sa, b, sb, dtype))
    assert torch.equal(got, kr.byte_matmul(a, sa, b, sb, dtype=dtype))
