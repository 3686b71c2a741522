"""One tensor as several arguments of an operator, or of several: its gradient is the sum of theirs.

Tolerances.  The gradients that are added are the operator's own; torch adds two of a type in 32 bits and
rounds once, three one after the other: whatever the order, off by an ulp, eps, of the terms' magnitudes for each
addition."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def normal(*shape, seed, dtype):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def near(got, parts):
    want, size = sum(p.double() for p in parts), sum(p.double().abs() for p in parts)
    off = torch.finfo(got.dtype).eps * (len(parts) - 1) * size
    assert bool(((got.double() - want).abs() <= off).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_layer_norm(kr, dtype, p):
    """x as its own residual, the weight as the bias, the sum used twice."""
    x, w = normal(9, 72, seed=1, dtype=dtype), normal(72, seed=2, dtype=dtype)
    d, ds = normal(9, 72, seed=3, dtype=dtype), normal(9, 72, seed=4, dtype=dtype)
    drop = dict(p=p, seed=5, offset=6)
    xg, wg = x.clone().requires_grad_(), w.clone().requires_grad_()
    n = kr.add_layer_norm(xg, wg, wg, xg, **drop)
    torch.autograd.backward([n.out, n.sum], [d, ds])
    m = kr.add_layer_norm(x, w, w, x, **drop)
    dx, dres, dw, db = kr.add_layer_norm_backward(d, m.sum, w, m.mean, m.rstd, ds, **drop)
    near(xg.grad, [dx, dres])
    near(wg.grad, [dw.to(dtype), db.to(dtype)])


@pytest.mark.parametrize("p", [0.0, 0.4, 1.0])
def test_dropout(kr, p):
    x, d = normal(9, 72, seed=1, dtype=torch.bfloat16), normal(9, 72, seed=3, dtype=torch.bfloat16)
    xg = x.clone().requires_grad_()
    kr.dropout(xg, p, 5, 6, xg).backward(d)
    near(xg.grad, [kr.dropout(d, p, 5, 6), d])


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_linear(kr, dtype):
    """A square matrix times its own transpose, and a weight of two layers."""
    x, d = normal(72, 72, seed=1, dtype=dtype), normal(72, 72, seed=2, dtype=dtype)
    g = x.clone().requires_grad_()
    kr.scaled_linear(g, g).backward(d)
    near(g.grad, kr.scaled_linear_backward(d, x, x))
    w = normal(72, 72, seed=3, dtype=dtype)
    g = w.clone().requires_grad_()
    h = kr.scaled_linear(x, g)
    kr.scaled_linear(h, g).backward(d)
    dh, two = kr.scaled_linear_backward(d, h.detach(), w)
    _, one = kr.scaled_linear_backward(dh, x, w)
    near(g.grad, [one, two])
