"""What the operators on values held in 8-bit floating point refuse: the C ABI on the host, before any
launch; the binding on tensors of another type or shape."""

import ctypes

import pytest
import torch

from paper_2601_17654_amd import binding as b

L = b._lib
BF16, F32 = 2, 0


def scaled(q=16, ld=304, room=304, scale=16, lds=128):
    return b.KrScaled(q, ld, room, scale, lds)


def hold(type=BF16, rows=100, width=300, x=16, ldx=300, square=0, plain=scaled(),
         crossed=scaled(16, 112, 112, 16, 384)):
    return L.kr_scaled_hold(type, rows, width, x, ldx, square, plain, crossed, None)


@pytest.mark.parametrize("bad", [
    dict(type=3), dict(rows=-1), dict(width=0), dict(x=None), dict(x=17), dict(ldx=299), dict(square=2),
    dict(plain=None, crossed=None), dict(plain=scaled(q=0)), dict(plain=scaled(ld=303)),
    dict(plain=scaled(room=299)), dict(plain=scaled(room=385, ld=400)), dict(plain=scaled(scale=0)),
    dict(plain=scaled(scale=18)), dict(plain=scaled(lds=127)), dict(plain=scaled(lds=130)),
    dict(crossed=scaled(16, 112, 112, 16, 380)), dict(crossed=scaled(16, 112, 99, 16, 384)),
    dict(crossed=scaled(16, 200, 129, 16, 384))])
def test_hold(bad):
    assert hold(**bad) == b.KR_EINVAL


def test_hold_sizes():
    assert hold(rows=0, x=None) == b.KR_OK
    big = (1 << 30) + 1
    assert hold(rows=big) == b.KR_EUNSUPPORTED
    assert hold(width=big, ldx=big) == b.KR_EUNSUPPORTED
    assert hold(rows=1 << 21, width=1 << 20, ldx=1 << 20) == b.KR_EUNSUPPORTED


@pytest.mark.parametrize("bad", [
    dict(type=-1), dict(rows=-1), dict(width=0), dict(h=None), dict(h=scaled(q=0)), dict(out=None),
    dict(out=17), dict(ldo=299), dict(h=scaled(lds=126))])
def test_values(bad):
    v = dict(type=BF16, rows=100, width=300, h=scaled(), out=16, ldo=300)
    assert L.kr_scaled_values(*{**v, **bad}.values(), None) == b.KR_EINVAL
    assert L.kr_scaled_values(BF16, 0, 300, scaled(q=0, scale=0), None, 0, None) == b.KR_OK


def product(m=100, n=50, k=300, a=scaled(), bb=scaled()):
    return b.KrScaledProduct(m, n, k, a, bb)


BAD = [dict(m=-1), dict(n=0), dict(k=0), dict(a=scaled(q=0)), dict(bb=scaled(q=0)), dict(k=305),
       dict(a=scaled(ld=303)), dict(a=scaled(scale=0)), dict(bb=scaled(scale=2)), dict(m=129),
       dict(n=129), dict(a=scaled(lds=129))]


@pytest.mark.parametrize("bad", BAD)
def test_matmul(bad):
    p = product(**bad)
    assert L.kr_scaled_matmul_workspace(p) == 0
    assert L.kr_scaled_matmul(p, F32, 16, 4096, 16, 1 << 40, None) == b.KR_EINVAL


def test_matmul_arguments():
    p = product()
    need = L.kr_scaled_matmul_workspace(p)
    assert L.kr_scaled_matmul(None, F32, 16, 50, 16, 1 << 30, None) == b.KR_EINVAL
    for type, out, ldo, ws in ((3, 16, 50, 16), (F32, None, 50, 16), (F32, 18, 50, 16),
                               (F32, 16, 49, 16), (F32, 16, 50, 24)):
        assert L.kr_scaled_matmul(p, type, out, ldo, ws, 1 << 30, None) == b.KR_EINVAL
    if need:
        assert L.kr_scaled_matmul(p, F32, 16, 50, 16, need - 1, None) == b.KR_ECAPACITY
        assert L.kr_scaled_matmul(p, F32, 16, 50, None, need, None) == b.KR_ECAPACITY
    none = product(m=0, a=scaled(q=0, scale=0))
    assert L.kr_scaled_matmul(none, F32, None, 0, None, 0, None) == b.KR_OK
    wide = dict(ld=1 << 22, room=1 << 22)
    big = product(k=(1 << 21) + 1, a=scaled(**wide), bb=scaled(**wide))
    assert L.kr_scaled_matmul(big, F32, 16, 50, 16, 1 << 30, None) == b.KR_EUNSUPPORTED
    rows = scaled(lds=1 << 31)
    for more in (dict(m=1 << 31, a=scaled(lds=1 << 31)), dict(n=(1 << 27) + 1, bb=rows),
                 dict(m=1 << 22, n=1 << 21, a=rows, bb=rows)):
        assert L.kr_scaled_matmul(product(**more), F32, 16, 1 << 28, 16, 1 << 30,
                                  None) == b.KR_EUNSUPPORTED


def test_binding():
    q = torch.zeros(4, 300).to(torch.float8_e4m3fn)
    scale = torch.zeros(3, 128, dtype=torch.uint8)
    good = b.Scaled(q, scale)
    k, rows, width, _ = b._held(good, "h", -1)
    assert (rows, width, k.ld, k.room, k.lds) == (4, 300, 300, 300, 128)
    for bad, error in (
            (q, TypeError), (b.Scaled(q.float(), scale), TypeError),
            (b.Scaled(q, scale.int()), TypeError), (b.Scaled(q, scale[:2]), ValueError),
            (b.Scaled(q, scale[:, :127]), ValueError), (b.Scaled(q, scale[0]), ValueError),
            (b.Scaled(q, scale, 304), ValueError), (b.Scaled(q[:, :290], scale, 301), ValueError)):
        with pytest.raises(error):
            b._held(bad, "h", -1)
    x = torch.zeros(4, 300)
    for call in (lambda: b.scaled_hold(x.double()), lambda: b.scaled_hold([1.0]),
                 lambda: b.scaled_values(x), lambda: b.scaled_values(good, torch.int8),
                 lambda: b.scaled_matmul(x, good), lambda: b.scaled_matmul(good, good, torch.float64),
                 lambda: b.scaled_linear(x, x.half()), lambda: b.scaled_linear(x.long(), x.long())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: b.scaled_hold(x), lambda: b.scaled_matmul(good, good),
                 lambda: b.scaled_linear(x, x[:, :299]), lambda: b.scaled_linear(x, x[0]),
                 lambda: b.scaled_linear(x, x), lambda: b.scaled_linear_backward(x, x, x[:, 1:])):
        with pytest.raises(ValueError):
            call()


def test_one_row_with_room():
    """A single row keeps the room that its storage has."""
    store = torch.zeros(1, 304).to(torch.float8_e4m3fn)
    scale = torch.zeros(3, 128, dtype=torch.uint8)
    k = b._held(b.Scaled(store[:, :300], scale, 304), "h", -1)[0]
    assert (k.ld, k.room) == (304, 304)


def linear(**bad):
    v = dict(type=BF16, rows=40, width=72, hidden=56, x=16, w=16, ldx=72, ldw=72)
    return b.KrLinear(*{**v, **bad}.values())


LINEAR_BAD = [dict(type=3), dict(rows=-1), dict(width=0), dict(hidden=0), dict(x=0), dict(w=0), dict(x=17),
              dict(w=17), dict(ldx=71), dict(ldw=71)]


@pytest.mark.parametrize("bad", LINEAR_BAD)
def test_linear(bad):
    l = linear(**bad)
    assert L.kr_scaled_linear_workspace(l) == 0 and L.kr_scaled_linear_backward_workspace(l) == 0
    assert L.kr_scaled_linear(l, 16, 56, 16, 1 << 30, None) == b.KR_EINVAL
    assert L.kr_scaled_linear_backward(l, 16, 56, 16, 72, 16, 72, 16, 1 << 30, None) == b.KR_EINVAL


def test_linear_arguments():
    l = linear()
    need, back = L.kr_scaled_linear_workspace(l), L.kr_scaled_linear_backward_workspace(l)
    # the operands, a byte a value and a byte for each block of a row
    assert need >= 40 * 80 + 128 + 56 * 80 + 128 and back >= 2 * (40 * 64 + 72 * 64)
    for out, ldo, ws in ((None, 56, 16), (17, 56, 16), (16, 55, 16), (16, 56, 24)):
        assert L.kr_scaled_linear(l, out, ldo, ws, need, None) == b.KR_EINVAL
    assert L.kr_scaled_linear(l, 16, 56, 16, need - 1, None) == b.KR_ECAPACITY
    assert L.kr_scaled_linear(l, 16, 56, None, need, None) == b.KR_ECAPACITY
    good = [16, 56, 16, 72, 16, 72, 16, back]
    for at, value, says in ((0, None, b.KR_EINVAL), (0, 17, b.KR_EINVAL), (1, 55, b.KR_EINVAL),
                            (2, 17, b.KR_EINVAL), (3, 71, b.KR_EINVAL), (4, 17, b.KR_EINVAL),
                            (5, 71, b.KR_EINVAL), (6, 24, b.KR_EINVAL), (6, None, b.KR_ECAPACITY),
                            (7, back - 1, b.KR_ECAPACITY)):
        bad = list(good)
        bad[at] = value
        assert L.kr_scaled_linear_backward(l, *bad, None) == says, (at, value)
    none = linear(rows=0, x=0)
    assert L.kr_scaled_linear(none, None, 0, None, 0, None) == b.KR_OK
    assert L.kr_scaled_linear_backward(none, None, 0, None, 0, None, 0, None, 0, None) == b.KR_OK
    wide = linear(width=(1 << 21) + 1, ldx=1 << 22, ldw=1 << 22)
    assert L.kr_scaled_linear(wide, 16, 56, 16, 1 << 40, None) == b.KR_EUNSUPPORTED
    tall = linear(rows=(1 << 21) + 1)
    assert L.kr_scaled_linear_workspace(tall) > 0 and L.kr_scaled_linear_backward_workspace(tall) == 0
    assert L.kr_scaled_linear_backward(tall, *good, None) == b.KR_EUNSUPPORTED
