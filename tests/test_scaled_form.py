"""The tests' own form of held values, on the CPU: its rounding against torch's conversion, its scale
against its definition."""

import pytest
import torch

from tests.scaled_form import e4m3, hold, in_order, values


def test_rounding():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    every = every[torch.isfinite(every)].sort().values.unique()
    assert torch.equal(e4m3(every), every)
    halves = (every[1:] + every[:-1]) / 2
    near = torch.cat([halves, halves * (1 + 2.0 ** -20), halves * (1 - 2.0 ** -20)])
    assert torch.equal(e4m3(near), near.float().to(torch.float8_e4m3fn).double())


@pytest.mark.parametrize("top,e", [(448.0, 0), (449.0, 1), (1.0, -8), (0.875, -9), (0.876, -8),
                                   (2.0 ** -150, -127), (0.0, -127), (3e38, 120)])
def test_scale(top, e):
    x = torch.zeros(2, 130, dtype=torch.float64)
    x[0, 5] = -top
    q, byte = hold(x)
    assert byte.tolist() == [[e + 127, 0], [0, 0]]
    assert float((values(q, byte)[0, 5] + top).abs()) <= max(top * 2.0 ** -4, 2.0 ** -137)
    assert hold(x, True)[1].tolist() == [[e + 127, 0], [e + 127, 0]]


def test_order():
    byte = torch.randint(0, 256, (300, 3))
    got = in_order(byte)
    for i in range(300):
        assert got[2, i // 128 * 128 + i % 16 * 8 + i % 128 // 16] == byte[i, 2]
