"""Sizes whose weight gradients would take more blocks than a launch has: refused on the host, with
or without rows."""

import ctypes

import pytest

from paper_2601_17654_amd import binding as b

L = b._lib
one, null = ctypes.c_void_p(16), ctypes.c_void_p(0)


def gated(rows, width, hidden):
    ld = 1 << 20
    return b.KrGated(2, 0, rows, width, hidden, 16, 16, 16, ld, ld, ld)


# 2 hidden / 128 * width / 64 tiles of the gradients above 2^23, rows x either below
TOO_MANY = [(0, 1 << 20, 1 << 20), (40, 1 << 20, 1 << 20), (1, 1 << 20, (1 << 15) + 64),
            (300, (1 << 15) + 64, 1 << 20)]


@pytest.mark.parametrize("rows,width,hidden", TOO_MANY)
def test_refused(rows, width, hidden):
    p = ctypes.byref(gated(rows, width, hidden))
    assert L.kr_gated_projection_backward_workspace(p) == 0
    assert L.kr_gated_projection_backward(p, one, 1 << 20, one, 1 << 20, one, 1 << 20, one,
                                          1 << 20, one, 1 << 60, null) == b.KR_EUNSUPPORTED


@pytest.mark.parametrize("rows,width,hidden", [(40, 1 << 20, 1 << 15), (40, 1 << 15, 1 << 20)])
def test_largest(rows, width, hidden):
    """At the limit: taken (too small a workspace is found before any launch)."""
    p = ctypes.byref(gated(rows, width, hidden))
    need = L.kr_gated_projection_backward_workspace(p)
    assert need >= rows * 4 * hidden
    assert L.kr_gated_projection_backward(p, one, 1 << 20, one, 1 << 20, one, 1 << 20, one,
                                          1 << 20, one, need - 1, null) == b.KR_ECAPACITY
