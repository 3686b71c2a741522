"""What dropout and layer norm refuse: the C ABI answers on the host, before any launch; the binding
raises on values out of range and on tensors of another type."""

import ctypes

import pytest
import torch

from paper_2601_17654_amd import binding as b

L = b._lib
one, odd, null = ctypes.c_void_p(16), ctypes.c_void_p(17), ctypes.c_void_p(0)
BF16, F32 = 2, 0


def drop(p=0.1, at=None):
    return ctypes.byref(b.KrDrop(p, 1, 2, at))


def dropout(type=BF16, rows=4, width=8, x=one, ldx=8, res=one, ldr=8, d=drop(), out=one, ldo=8):
    return L.kr_dropout(type, rows, width, x, ldx, res, ldr, d, out, ldo, null)


@pytest.mark.parametrize("bad", [
    dict(type=3), dict(type=-1), dict(rows=-1), dict(width=0), dict(x=null), dict(x=odd), dict(ldx=7),
    dict(res=odd), dict(ldr=7), dict(out=null), dict(out=odd), dict(ldo=7), dict(d=None),
    dict(d=drop(-0.1)), dict(d=drop(1.1)), dict(d=drop(float("nan"))), dict(d=drop(0.1, 4))])
def test_dropout(bad):
    assert dropout(**bad) == b.KR_EINVAL


def test_dropout_sizes():
    big = 1 << 33
    assert dropout(rows=(1 << 32) + 1) == b.KR_EUNSUPPORTED
    assert dropout(width=(1 << 30) + 1, ldx=big, ldr=big, ldo=big) == b.KR_EUNSUPPORTED
    assert dropout(rows=0, x=null, out=null) == b.KR_OK


def norm(type=BF16, rows=4, width=8, x=one, ldx=8, res=one, ldr=8, w=one, bias=one, eps=1e-5,
         d=drop(), sum=one, lds=8, out=one, ldo=8):
    return L.kr_add_layer_norm(type, rows, width, x, ldx, res, ldr, w, bias, eps, d, sum, lds, out,
                               ldo, null, null, null)


@pytest.mark.parametrize("bad", [
    dict(type=3), dict(rows=-1), dict(width=0), dict(x=null), dict(w=null), dict(out=null),
    dict(ldx=7), dict(ldr=7), dict(lds=7), dict(ldo=7), dict(eps=-1.0), dict(eps=float("nan")),
    dict(eps=float("inf")), dict(x=odd), dict(res=odd), dict(w=odd), dict(bias=odd), dict(sum=odd),
    dict(out=odd), dict(d=drop(2.0)), dict(d=drop(float("nan")))])
def test_norm(bad):
    assert norm(**bad) == b.KR_EINVAL


def test_norm_sizes():
    big = 1 << 26
    assert norm(width=(1 << 24) + 1, ldx=big, ldr=big, lds=big, ldo=big) == b.KR_EUNSUPPORTED
    assert norm(rows=(1 << 32) + 1) == b.KR_EUNSUPPORTED
    assert norm(rows=0, x=null, w=null, out=null) == b.KR_OK


def test_norm_backward():
    need = L.kr_add_layer_norm_backward_workspace(F32, 100, 8)
    assert need >= 64 and need % 64 == 0
    assert L.kr_add_layer_norm_backward_workspace(F32, 100, 0) == 0
    assert L.kr_add_layer_norm_backward_workspace(7, 100, 8) == 0
    two = ctypes.c_void_p(32)
    args = [F32, 100, 8, one, 8, one, 8, one, one, one, null, 0, drop(), one, 8, two, 8, one, one, one,
            need, null]
    for at, value, says in (
            (0, 5, b.KR_EINVAL), (1, -1, b.KR_EINVAL), (2, 0, b.KR_EINVAL), (3, null, b.KR_EINVAL),
            (4, 7, b.KR_EINVAL), (5, null, b.KR_EINVAL), (6, 7, b.KR_EINVAL), (7, null, b.KR_EINVAL),
            (8, null, b.KR_EINVAL), (9, null, b.KR_EINVAL), (10, odd, b.KR_EINVAL),
            (12, drop(-1.0), b.KR_EINVAL), (13, null, b.KR_EINVAL), (14, 7, b.KR_EINVAL),
            (15, null, b.KR_EINVAL), (15, one, b.KR_EINVAL), (16, 7, b.KR_EINVAL),
            (17, null, b.KR_EINVAL), (19, odd, b.KR_EINVAL), (19, null, b.KR_ECAPACITY),
            (20, need - 1, b.KR_ECAPACITY), (1, (1 << 32) + 1, b.KR_EUNSUPPORTED)):
        bad = list(args)
        bad[at] = value
        assert L.kr_add_layer_norm_backward(*bad) == says, (at, value)


@pytest.mark.parametrize("bad", [dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(seed=-1),
                                 dict(seed=1 << 64), dict(offset=-1), dict(offset=1 << 64),
                                 dict(seed=torch.zeros(2, dtype=torch.int64))])
def test_binding_values(bad):
    with pytest.raises(ValueError):
        b._drop(**{**dict(p=0.1, seed=0, offset=0, dev=-1), **bad})


def test_binding_types():
    x = torch.zeros(2, 8)
    with pytest.raises(TypeError):
        b._drop(0.1, torch.zeros(1), 0, -1)
    with pytest.raises(TypeError):
        b.dropout(x.double(), 0.1, 0)
    with pytest.raises(TypeError):
        b.add_layer_norm([1.0], x[0])
    with pytest.raises(TypeError):
        b.add_layer_norm_backward(x.long(), x, x[0], x[:, 0], x[:, 0])
    with pytest.raises(ValueError):
        b.dropout(x, 0.1, 0)  # not on the device
