"""The product's form of few rows takes 16: of more it would put sums that it has no room for, and says so
on the host, before any launch."""

import ctypes

from paper_2601_17654_amd import binding as b

INVALID_VALUE = 1  # hipErrorInvalidValue


class Held(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("ld", ctypes.c_int64), ("bytes", ctypes.c_int64),
                ("scale", ctypes.c_void_p), ("lds", ctypes.c_int64)]


class Args(ctypes.Structure):
    _fields_ = [("out_type", ctypes.c_int), ("m", ctypes.c_int64), ("n", ctypes.c_int64),
                ("k", ctypes.c_int64), ("a", Held), ("b", Held), ("out", ctypes.c_void_p),
                ("ldo", ctypes.c_int64), ("part", ctypes.c_void_p)]


def test_more_than_sixteen():
    few = getattr(b._lib, "_ZN2kr17launch_scaled_fewERKNS_10ScaledArgsEP12ihipStream_t")
    h = Held(16, 128, 128, 16, 128)
    for m in (17, 32, 1 << 20):
        for out_type in (0, 1, 2):
            assert few(ctypes.byref(Args(out_type, m, 64, 128, h, h, 16, 64, None)), None) == INVALID_VALUE
