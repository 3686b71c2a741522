"""How rows are dealt to blocks and launches (kr_dealt.h, plain C++): a launch's grid has fewer than 2^32
threads and its blocks hold its rows, at every width that dropout and the values of a held matrix take."""

import ctypes
import os
import random
import subprocess

import pytest

from tests.dealt import dealt, rows_a_launch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r'''
#include "kr_dealt.h"
extern "C" void cut(int64_t groups, int64_t rows, int64_t *to)
{
    const kr::Dealt s = kr::dealt(groups);
    to[0] = s.log_tpr;
    to[1] = s.groups;
    to[2] = s.chunks;
    to[3] = kr::dealt_rows(s);
    to[4] = kr::dealt_blocks(s, rows);
}
'''


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    at = tmp_path_factory.mktemp("dealt")
    (at / "cut.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                           os.path.join(ROOT, "paper_2601_17654_amd", "csrc"), "-o",
                           str(at / "cut.so"), str(at / "cut.cpp")])
    lib = ctypes.CDLL(str(at / "cut.so"))
    lib.cut.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.POINTER(ctypes.c_int64)]

    def call(groups, rows=1):
        to = (ctypes.c_int64 * 5)()
        lib.cut(groups, rows, to)
        return dict(zip(("log", "groups", "chunks", "rows", "blocks"), to))

    return call


def widths():
    rng = random.Random(1)
    for b in range(31):
        yield from {max(1, (1 << b) - 1), 1 << b, min(1 << 30, (1 << b) + 1)}
        for _ in range(30):
            yield rng.randint(1 << b, min(1 << 30, 2 << b))


# neighbours of a thread: dropout's, those of values in 32 and in 16 bits
@pytest.mark.parametrize("group", [8, 4, 16])
def test_grids(cut, group):
    for width in widths():
        groups = -(-width // group)
        s = cut(groups)
        assert s["groups"] == groups and s["chunks"] << s["log"] >= groups
        assert (s["log"], s["chunks"]) == dealt(groups) and s["rows"] == rows_a_launch(groups)
        side = 256 >> s["log"]  # rows of a block
        for rows in (1, side, side + 1, 128, 1000, s["rows"] - 1, s["rows"]):
            if not 1 <= rows <= s["rows"]:
                continue
            blocks = cut(groups, rows)["blocks"]
            assert blocks * 256 < 1 << 32, (width, rows)
            assert blocks % s["chunks"] == 0 and blocks // s["chunks"] * side >= rows


def test_wide_rows_go_in_fewer_than_128_a_launch(cut):
    """Where 128 rows have 2^32 threads and more: values in 32 bits of 2^27 columns, in 16 bits of 2^29."""
    for group, width in ((4, 1 << 27), (16, 1 << 29), (16, 1 << 30)):
        s = cut(width // group)
        assert cut(width // group, 128)["blocks"] * 256 >= 1 << 32
        assert 1 <= s["rows"] < 128
