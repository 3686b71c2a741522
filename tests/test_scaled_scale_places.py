"""A held matrix's scale bytes wherever a tensor has them: at an odd address, in rows of an odd length or in odd
columns they are copied to where the kernels can read them."""

import ctypes

import pytest
import torch

from paper_2601_17654_amd import binding as b


def scales():
    bytes_ = torch.arange(3 * 256).remainder(251).to(torch.uint8).view(3, 256)
    yield "as they are", 256, bytes_
    for at in (1, 2, 3):  # contiguous, which a copy that only makes it so leaves where it is
        flat = torch.zeros(3 * 256 + 8, dtype=torch.uint8)
        moved = flat[4 - flat.data_ptr() % 4 + at:][:3 * 256].view(3, 256)
        yield "at an odd address", 256, moved.copy_(bytes_)
    wide = torch.zeros(3, 259, dtype=torch.uint8)
    wide[:, :256] = bytes_
    yield "in rows of an odd length", 256, wide
    yield "every second", 256, bytes_.repeat_interleave(2, 1)[:, ::2]
    yield "crossed", 256, bytes_.t().contiguous().t()
    one = torch.zeros(129, dtype=torch.uint8)
    one[1:] = bytes_[0, :128]
    yield "a row with a step of its own", 128, one.as_strided((1, 128), (3, 1), 1)


@pytest.mark.parametrize("case", range(8))
def test_read_where_the_kernels_can(case):
    what, rows, s = list(scales())[case]
    width = 128 * s.shape[0]
    q = torch.zeros(rows - 5, width).to(torch.float8_e4m3fn)
    k, n, w, keep = b._held(b.Scaled(q, s), "h", -1)
    assert (n, w) == (rows - 5, width)
    assert k.scale % 4 == 0 and k.lds % 4 == 0 and k.lds >= rows, what
    for block in range(s.shape[0]):
        read = ctypes.string_at(k.scale + block * k.lds, rows)
        assert list(read) == s[block, :rows].tolist(), what
