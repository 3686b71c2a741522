"""The smoke check of layer norm, dropout and the 8-bit float products finds a wrong result: it is run here,
on the CPU, with plain operators in their place, as they are and with one mistake each."""

import types

import pytest
import torch

import __graft_entry__ as entry
from tests.philox import factor
from tests.scaled_form import hold, values

bf = torch.bfloat16


class Plain:
    def __init__(self, mistake=""):
        self.mistake = mistake

    def add_layer_norm(self, x, w, b, r):
        s = x.float() + r.float()
        m = 0 * s[:, :1] if self.mistake == "mean" else s.mean(-1, keepdim=True)
        f = 1 / ((s - m).square().mean(-1, keepdim=True) + 1e-5).sqrt()
        n = (s - m) * f * w.float() + (0 if self.mistake == "bias" else b.float())
        return types.SimpleNamespace(out=n.to(bf), sum=(x if self.mistake == "sum" else s).to(bf),
                                     mean=m[:, 0], rstd=f[:, 0])

    def scaled_hold(self, x, square=False, plain=True, crossed=False):
        v = values(*hold(x.t() if crossed else x, square))
        if self.mistake == "held":
            v = v * 1.07
        return types.SimpleNamespace(plain=v, crossed=v)

    def scaled_values(self, v, dtype):
        return v.to(dtype)

    def _values(self, x, square=False):
        return values(*hold(x, square))

    def scaled_linear(self, x, w):
        y = self._values(x) @ self._values(w, True).t()
        return (y * (1.02 if self.mistake == "linear" else 1)).to(bf)

    def scaled_linear_backward(self, d, x, w):
        dx = self._values(d) @ self._values(w.t(), True).t()
        dw = self._values(d.t()) @ self._values(x.t()).t()
        return (0 if self.mistake == "dx" else 1) * dx.to(bf), dw.to(bf)

    def add_layer_norm_backward(self, d, s, w, m, f, ds):
        h, t = (s.float() - m[:, None]) * f[:, None], d.float() * w.float()
        c0 = 0 if self.mistake == "level" else t.mean(-1, keepdim=True)
        c1 = 0 if self.mistake == "along" else (t * h).mean(-1, keepdim=True)
        dx = (f[:, None] * (t - c0 - h * c1) + (0 if self.mistake == "dsum" else ds.float())).to(bf)
        dw = (d.float() * (t if self.mistake == "dweight" else h)).sum(0)
        return dx, dx, dw, (h if self.mistake == "dbias" else d.float()).sum(0)

    def dropout(self, x, p, seed, offset=0):
        if self.mistake == "offset":
            offset = 0
        f = factor(*x.shape, p + (0.05 if self.mistake == "share" else 0), seed, offset).float()
        return x * f * (0.75 if self.mistake == "factor" else 1)


def test_right():
    entry._smoke_layer_norm_block(Plain(), torch, "cpu")


@pytest.mark.parametrize("mistake", ["mean", "bias", "sum", "held", "linear", "dx", "level", "along",
                                     "dsum", "dweight", "dbias", "offset", "share", "factor"])
def test_mistakes(mistake):
    with pytest.raises(AssertionError):
        entry._smoke_layer_norm_block(Plain(mistake), torch, "cpu")
