"""The tests' generator against the known answers that are published for it, and the share of values that
it keeps."""

import pytest

from tests.philox import factor, philox

KNOWN = [
    ([0] * 4, [0] * 2, [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
    ([0xffffffff] * 4, [0xffffffff] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
    ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0],
     [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]),
]


@pytest.mark.parametrize("counter,key,words", KNOWN)
def test_known_answers(counter, key, words):
    assert [int(x) for x in philox(counter, key)] == words


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999, 1.0])
def test_share(p):
    n = 512 * 1024
    kept = float((factor(512, 1024, p, 7, 3) > 0).double().mean())
    assert abs(kept - (1 - p)) <= 2 ** -17 + 5 * (p * (1 - p) / n) ** 0.5  # five deviations
