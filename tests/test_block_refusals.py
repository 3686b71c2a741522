"""What the transformer-block operators refuse: the C ABI answers on the host, before any
launch; the binding raises on tensors of another type, shape or device."""

import ctypes

import pytest
import torch

from paper_2601_17654_amd import binding as b

L = b._lib
one = ctypes.c_void_p(16)
odd = ctypes.c_void_p(17)
null = ctypes.c_void_p(0)
BF16, F32 = 2, 0


def norm(type=BF16, rows=4, width=8, x=one, ldx=8, res=one, ldr=8, w=one, eps=1e-6, sum=one,
         lds=8, out=one, ldo=8):
    return L.kr_add_rms_norm(type, rows, width, x, ldx, res, ldr, w, eps, sum, lds, out, ldo, null,
                             null)


@pytest.mark.parametrize("bad", [
    dict(type=3), dict(type=-1), dict(rows=-1), dict(width=0), dict(x=null), dict(w=null),
    dict(out=null), dict(ldx=7), dict(ldr=7), dict(lds=7), dict(ldo=7), dict(eps=-1.0),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(x=odd), dict(res=odd), dict(w=odd),
    dict(sum=odd), dict(out=odd)])
def test_norm(bad):
    assert norm(**bad) == b.KR_EINVAL


def test_norm_sizes():
    assert norm(width=(1 << 30) + 1, ldx=1 << 31, ldr=1 << 31, lds=1 << 31,
                ldo=1 << 31) == b.KR_EUNSUPPORTED
    assert norm(rows=0, x=null, w=null, out=null) == b.KR_OK


def test_norm_bytes():
    args = [BF16, 4, 8, one, 8, null, 0, one, 1e-6, null, 0, odd, 8, one, null, null]
    for at, value in ((3, null), (11, null), (13, null), (12, 7), (1, -1), (2, 0), (0, 9)):
        bad = list(args)
        bad[at] = value
        assert L.kr_add_rms_norm_bytes(*bad) == b.KR_EINVAL


def test_norm_backward():
    need = L.kr_add_rms_norm_backward_workspace(F32, 100, 8)
    assert need >= 32 and need % 32 == 0
    assert L.kr_add_rms_norm_backward_workspace(F32, 100, 0) == 0
    assert L.kr_add_rms_norm_backward_workspace(7, 100, 8) == 0
    args = [F32, 100, 8, one, 8, one, 8, one, one, null, 0, one, 8, one, one, need, null]
    short = list(args)
    short[15] = need - 1
    assert L.kr_add_rms_norm_backward(*short) == b.KR_ECAPACITY
    for at, value in ((0, 5), (1, -1), (2, 0), (3, null), (4, 7), (5, null), (6, 7), (7, null),
                      (8, null), (9, odd), (11, null), (12, 7), (13, null), (14, odd)):
        bad = list(args)
        bad[at] = value
        assert L.kr_add_rms_norm_backward(*bad) == b.KR_EINVAL, at


def test_binding_types():
    x = torch.zeros(2, 8)
    with pytest.raises(TypeError):
        b.add_rms_norm(x.double(), x[0].double())
    with pytest.raises(TypeError):
        b.add_rms_norm([1.0], x[0])
    with pytest.raises(TypeError):
        b.add_rms_norm_backward(x.long(), x, x[0], x[:, 0])
