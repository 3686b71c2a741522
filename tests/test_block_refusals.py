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


def gated(**bad):
    v = dict(type=BF16, act=0, rows=4, width=8, hidden=8, x=16, wg=16, wu=16, ldx=8, ldg=8, ldu=8)
    v.update(bad)
    return b.KrGated(*v.values())


GATED_BAD = [dict(type=0), dict(type=3), dict(act=2), dict(act=-1), dict(rows=-1), dict(width=0),
             dict(hidden=0), dict(x=0), dict(wg=0), dict(wu=0), dict(x=17), dict(wg=17), dict(wu=17),
             dict(ldx=7), dict(ldg=7), dict(ldu=7)]
GATED_BIG = [dict(rows=1 << 31), dict(width=(1 << 20) + 1, ldx=1 << 21, ldg=1 << 21, ldu=1 << 21),
             dict(hidden=(1 << 20) + 1)]


def test_gated():
    fwd, back = L.kr_gated_projection, L.kr_gated_projection_backward
    big = 1 << 40

    def both(g, ldo=1 << 21, ws=one, nbytes=big, out=one):
        p = ctypes.byref(g)
        return {fwd(p, out, ldo, ws, nbytes, null),
                back(p, one, ldo, one, ldo, out, ldo, one, ldo, ws, nbytes, null)}

    for bad in GATED_BAD:
        assert both(gated(**bad)) == {b.KR_EINVAL}, bad
        assert L.kr_gated_projection_workspace(ctypes.byref(gated(**bad))) == 0
        assert L.kr_gated_projection_backward_workspace(ctypes.byref(gated(**bad))) == 0
    for bad in GATED_BIG:
        assert both(gated(**bad)) == {b.KR_EUNSUPPORTED}, bad
    assert both(gated(), out=null) == {b.KR_EINVAL}
    assert both(gated(), out=odd) == {b.KR_EINVAL}
    assert both(gated(), ldo=7) == {b.KR_EINVAL}
    assert both(gated(), ws=odd) == {b.KR_EINVAL}
    assert fwd(None, one, 8, one, big, null) == b.KR_EINVAL
    assert fwd(ctypes.byref(gated(rows=0, x=0)), null, 0, null, 0, null) == b.KR_OK
    g = gated(rows=40, width=9, ldx=9, ldg=9, ldu=9)  # rows of 18 bytes: copies in the workspace
    need = L.kr_gated_projection_workspace(ctypes.byref(g))
    assert need >= (40 + 8 + 8) * 32
    assert fwd(ctypes.byref(g), one, 8, one, need - 1, null) == b.KR_ECAPACITY
    assert fwd(ctypes.byref(g), one, 8, null, need, null) == b.KR_ECAPACITY
    need = L.kr_gated_projection_backward_workspace(ctypes.byref(gated()))
    assert need >= 4 * 2 * 8 * 2
    assert back(ctypes.byref(gated()), one, 8, one, 8, one, 8, one, 8, one, need - 1,
                null) == b.KR_ECAPACITY


def test_bytes():
    def args(**bad):
        v = dict(m=4, n=8, k=16, a=16, b=16, lda=16, ldb=16, sa=16, sb=16)
        v.update(bad)
        return ctypes.byref(b.KrBytes(*v.values()))

    call = L.kr_byte_matmul
    for bad in (dict(m=-1), dict(n=0), dict(k=0), dict(a=0), dict(b=0), dict(lda=15), dict(ldb=15),
                dict(sa=0), dict(sb=0)):
        assert call(args(**bad), BF16, one, 8, one, 1 << 40, null) == b.KR_EINVAL, bad
        assert L.kr_byte_matmul_workspace(args(**bad)) == 0
    for bad in (dict(k=131072, lda=1 << 18, ldb=1 << 18), dict(m=1 << 31), dict(n=(1 << 30) + 1)):
        assert call(args(**bad), BF16, one, 1 << 31, one, 1 << 40, null) == b.KR_EUNSUPPORTED, bad
    assert call(args(), 3, one, 8, one, 1 << 40, null) == b.KR_EINVAL
    assert call(args(), BF16, null, 8, one, 1 << 40, null) == b.KR_EINVAL
    assert call(args(), BF16, one, 7, one, 1 << 40, null) == b.KR_EINVAL
    assert call(args(), F32, ctypes.c_void_p(18), 8, one, 1 << 40, null) == b.KR_EINVAL
    assert call(None, F32, one, 8, one, 1 << 40, null) == b.KR_EINVAL
    assert call(args(m=0, a=0, sa=0), F32, null, 0, null, 0, null) == b.KR_OK
    bad = args(m=40, k=17, lda=17, ldb=17)
    need = L.kr_byte_matmul_workspace(bad)
    assert need >= 48 * 32 and call(bad, F32, one, 8, one, need - 1, null) == b.KR_ECAPACITY


def test_binding_products():
    x, w = torch.zeros(2, 8), torch.zeros(4, 8)
    with pytest.raises(TypeError):
        b.gated_projection(x, w, w)  # 32-bit inputs
    with pytest.raises(TypeError):
        b.byte_matmul(x, x[:, 0], w, w[:, 0])
    with pytest.raises(TypeError):
        b.byte_matmul(x.to(torch.int8), x[:, 0], w.to(torch.int8), w[:, 0], dtype=torch.float64)
    with pytest.raises(ValueError):
        b.gated_projection(x.half(), w.half(), w.half(), act="relu")
    with pytest.raises(ValueError):
        b.gated_projection(x.half(), w.half(), w.half())  # not on the device


def test_grids():
    """Sizes within each limit whose output would take more blocks than a launch has."""
    big = 1 << 20
    g = gated(rows=1 << 24, hidden=big, ldx=8)
    p = ctypes.byref(g)
    assert L.kr_gated_projection(p, one, big, one, 1 << 50, null) == b.KR_EUNSUPPORTED
    assert L.kr_gated_projection_backward(p, one, big, one, 8, one, 8, one, 8, one, 1 << 50,
                                          null) == b.KR_EUNSUPPORTED
    q = ctypes.byref(b.KrBytes(1 << 24, 1 << 24, 16, 16, 16, 16, 16, 16, 16))
    assert L.kr_byte_matmul(q, BF16, one, 1 << 24, one, 1 << 50, null) == b.KR_EUNSUPPORTED
    assert L.kr_byte_matmul_workspace(q) == 0
