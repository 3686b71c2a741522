"""The 8-bit product tiles' matrix instructions and direct copies, written as inline assembly like those of
the other products, keep the same distances from their neighbours (tests/test_matrix_instructions.py says
which): read off the built library."""

import glob
import os
import shutil
import subprocess

import pytest

from tests.test_matrix_instructions import LIB, OBJDUMP, faults, functions


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    assert os.path.exists(LIB), "the library is not built"
    at = str(tmp_path_factory.mktemp("code"))
    shutil.copy(LIB, os.path.join(at, "lib.so"))
    subprocess.check_call([OBJDUMP, "--offloading", "lib.so"], cwd=at, stdout=subprocess.DEVNULL)
    got = {}
    for path in glob.glob(os.path.join(at, "*gfx950")):
        with open(path, "rb") as f:
            if b"scaled_tile_kernel" not in f.read():
                continue
        got.update(functions(subprocess.check_output(
            [OBJDUMP, "-d", "--no-show-raw-insn", "--symbolize-operands", path], text=True)))
    return got


def test_tiles(kernels):
    tiles = {k: v for k, v in kernels.items() if "scaled_tile_kernel" in k}
    assert len(tiles) == 4  # two tile sizes, two types
    for name, code in tiles.items():
        # three bodies of a step (two in the loop, an odd last one)
        assert sum(x.mfma for x in code) in (3 * 16, 3 * 64), name
        assert all(x.op == "v_mfma_scale_f32_16x16x128_f8f6f4" for x in code if x.mfma), name
        assert sum(x.text.endswith(" lds") for x in code) in (5 * 9, 5 * 17), name
        found = list(faults(code))
        assert not found, "%s: %s" % (name, found[:5])


def test_wide_copies(kernels):
    """The compiler places that kernel's matrix instructions; its copies are written out."""
    wide = {k: v for k, v in kernels.items() if "scaled_wide_kernel" in k}
    assert len(wide) == 2  # two tile sizes
    for name, code in wide.items():
        assert sum(x.text.endswith(" lds") for x in code) in (3 * 9, 3 * 7)
        found = [f for f in faults(code) if "m0" in f]
        assert not found, found[:5]
