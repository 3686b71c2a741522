"""The smoke check of the block's operators finds a wrong result: it is run here, on the CPU, with plain
operators in 32 bits in the place of the kernels, as they are and with one mistake each."""

import types

import pytest
import torch

import __graft_entry__ as entry

bf = torch.bfloat16


class Plain:
    def __init__(self, mistake=""):
        self.mistake = mistake

    def add_rms_norm(self, x, w, r=None, eps=1e-6):
        s = x.float() + (r.float() if r is not None else 0)
        f = 1 / (s.square().mean(-1) + eps).sqrt()
        n = s * f[:, None] * (1 if self.mistake == "weight" else w.float())
        return types.SimpleNamespace(out=n.to(bf), sum=(x if self.mistake == "sum" else s).to(bf), rstd=f)

    def add_rms_norm_bytes(self, x, w, r=None, eps=1e-6):
        f = self.add_rms_norm(x, w, r, eps).rstd
        n = (x.float() + r.float()) * f[:, None] * w.float()
        scale = n.abs().amax(-1) / (120 if self.mistake == "scale" else 127)
        q = n / scale[:, None]
        q = q.trunc() if self.mistake == "trunc" else q.round()
        return types.SimpleNamespace(q=q.to(torch.int8), scale=scale)

    def add_rms_norm_backward(self, d, s, w, f, ds=None):
        h, t = s.float() * f[:, None], d.float() * w.float()
        c = 0 if self.mistake == "mean" else (t * h).mean(-1, keepdim=True)
        dx = f[:, None] * (t - h * c) + (0 if self.mistake == "dsum" else ds.float())
        return dx.to(bf), (0 if self.mistake == "dweight" else 1) * (d.float() * h).sum(0)

    def gated_projection(self, x, wg, wu):
        a, b = x.float() @ wg.float().t(), x.float() @ wu.float().t()
        return (torch.sigmoid(a) * a * b).to(bf)

    def gated_projection_backward(self, dh, x, wg, wu):
        a, b, d = x.float() @ wg.float().t(), x.float() @ wu.float().t(), dh.float()
        p = torch.sigmoid(a)
        slope = p if self.mistake == "slope" else p + a * p * (1 - p)
        dg, du = (d * b * slope).to(bf).float(), (d * a * p).to(bf).float()
        dx = dg @ wg.float() + (0 if self.mistake == "half" else du @ wu.float())
        got = [dx.to(bf), (dg.t() @ x.float()).to(bf), (du.t() @ x.float()).to(bf)]
        if self.mistake == "swapped":
            got[1], got[2] = got[2], got[1]
        if self.mistake == "zero":
            got[1] = got[1] * 0
        return got

    def byte_matmul(self, a, sa, b, sb, dtype):
        y = (a.double() @ b.double().t()).float()
        return y * (1 if self.mistake == "sa" else sa[:, None]) * sb


def test_right():
    entry._smoke_block(Plain(), torch, "cpu")


@pytest.mark.parametrize("mistake", ["weight", "sum", "scale", "trunc", "mean", "dsum", "dweight",
                                     "slope", "half", "swapped", "zero", "sa"])
def test_mistakes(mistake):
    with pytest.raises(AssertionError):
        entry._smoke_block(Plain(mistake), torch, "cpu")
