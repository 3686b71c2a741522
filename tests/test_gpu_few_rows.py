"""The form of few rows with four waves a block, which more than 8,176 outputs take, against 64
bits: the tolerances of the other tests of the same operators (the 8-bit product bit for bit)."""

import pytest
import torch

from tests import test_gpu_bytes as B
from tests import test_gpu_gated as G
from tests.test_gpu_block_tiles import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("width", [72, 1100, 2059])
@pytest.mark.parametrize("rows", [1, 2, 16, 17, 32])
def test_few_rows_many_outputs(kr, rows, width, dtype):
    """512 blocks or more take four waves each; widths that end before, in and after the loop of
    several steps."""
    print("few", rows, width, dtype, flush=True)
    hidden = 8205
    x, wg, wu, dh = inputs(rows, width, hidden, dtype)
    for act in ("silu", "gelu"):
        w = G.Want(x, wg, wu, dh, act, dtype)
        G.near(kr.gated_projection(x, wg, wu, act), w.h, w.eh, "h")


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("k", [100, 2059, 4200])
@pytest.mark.parametrize("m", [1, 16, 17, 20, 32])
def test_few_tokens_many_channels(kr, m, k, dtype):
    print("few bytes", m, k, dtype, flush=True)
    a, sa, b, sb = B.make(m, 8205, k, m + k)
    got = kr.byte_matmul(a, sa / k, b, sb, dtype=dtype)
    assert torch.equal(got, B.want(a, sa / k, b, sb, dtype))
