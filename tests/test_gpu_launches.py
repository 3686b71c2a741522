"""Rows past one launch: the values of a held matrix go on where the launch before ended, at either side of
its edge (tests/dealt.py says where that is)."""

import pytest
import torch

from tests.dealt import rows_a_launch
from tests.scaled_form import in_order

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


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
