"""How the tiled products cut their outputs: which of the tested shapes take large tiles and split
sums, and that a launch's grid holds every plan."""

import ctypes
import os
import random
import subprocess

import pytest

from tests.block_shapes import BYTES, GATED

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r'''
#include "kr_plan.h"
extern "C" void plan(int64_t m, int64_t n, int planes, int steps, int64_t *to)
{
    const kr::MmaPlan p = kr::mma_plan(m, n, planes, steps);
    to[0] = p.large;
    to[1] = p.tiles_m;
    to[2] = p.tiles_n;
    to[3] = p.splits;
    to[4] = p.per_split;
    to[5] = p.part_bytes;
}
'''


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                           os.path.join(ROOT, "paper_2601_17654_amd", "csrc"), "-o",
                           str(at / "plan.so"), str(at / "plan.cpp")])
    lib = ctypes.CDLL(str(at / "plan.so"))
    lib.plan.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                         ctypes.POINTER(ctypes.c_int64)]

    def call(m, n, planes, steps):
        to = (ctypes.c_int64 * 6)()
        lib.plan(m, n, planes, steps, to)
        return dict(zip(("large", "tiles_m", "tiles_n", "splits", "per", "part"), to))

    return call


def up(x, to):
    return -(-x // to)


def said(p):
    return bool(p["large"]), p["splits"] > 1


@pytest.mark.parametrize("shape", sorted(GATED))
def test_gated(plan, shape):
    rows, width, hidden = shape
    pad = up(hidden, 8) * 8
    k = up(up(2 * width, 16) * 16, 128)
    got = (plan(rows, pad, 2, k), plan(rows, width, 1, 2 * up(2 * pad, 128)),
           plan(2 * pad, width, 1, up(rows, 64)))
    assert tuple(map(said, got)) == GATED[shape]
    assert said(plan(rows, hidden, 2, k)) == GATED[shape][0]  # the forward product


@pytest.mark.parametrize("shape", sorted(BYTES))
def test_bytes(plan, shape):
    m, n, k = shape
    assert said(plan(m, n, 1, up(up(k, 16) * 16, 128))) == BYTES[shape]


def test_every_plan(plan):
    """Tiles and splits cover the product, no split is empty, and where the output has at most
    2^23 tiles of 128 x 64 the blocks' threads stay below 2^32."""
    rng = random.Random(1)

    def size(most):
        return int(2.0 ** rng.uniform(0, most))

    for _ in range(4000):
        m, n, planes, steps = size(31), size(27), rng.choice((1, 2)), rng.choice((0, size(15)))
        if up(m, 128) * up(n, 64) > 1 << 23:
            continue
        p = plan(m, n, planes, steps)
        tile = 256 if p["large"] else 128
        assert p["tiles_m"] == up(m, tile) and p["tiles_n"] == up(n, tile // planes)
        assert 1 <= p["splits"] <= 16 and p["per"] * p["splits"] >= steps
        assert steps == 0 or p["per"] * (p["splits"] - 1) < steps
        assert p["part"] == (4 * p["splits"] * planes * m * n if p["splits"] > 1 else 0)
        assert p["tiles_m"] * p["tiles_n"] * p["splits"] * 256 < 1 << 32
