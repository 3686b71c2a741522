"""The norm and the gated projection inside a graph of torch's: gradients reach every input by the
operators' own backward passes; what has no gradient says so."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def normal(*shape, seed, dtype=torch.bfloat16, grad=True):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(dtype).cuda().requires_grad_(grad)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_norm(kr, dtype):
    x, r = normal(2, 5, 72, seed=1, dtype=dtype), normal(2, 5, 72, seed=2, dtype=dtype)
    w = normal(72, seed=3, dtype=dtype)
    dout, dsum = (normal(2, 5, 72, seed=s, dtype=dtype, grad=False) for s in (4, 5))
    n = kr.add_rms_norm(x, w, r)
    assert n.out.requires_grad and n.sum.requires_grad and not n.rstd.requires_grad
    torch.autograd.backward([n.out, n.sum], [dout, dsum])
    with torch.no_grad():
        plain = kr.add_rms_norm(x, w, r)
        dx, dw = kr.add_rms_norm_backward(dout, plain.sum, w, plain.rstd, dsum)
    assert not plain.out.requires_grad and torch.equal(plain.out, n.out)
    assert torch.equal(plain.sum, n.sum) and torch.equal(plain.rstd, n.rstd)
    assert torch.equal(x.grad, dx) and torch.equal(r.grad, dx)
    assert w.grad.dtype == dtype and torch.equal(w.grad, dw.to(dtype))


def test_norm_by_one_path(kr):
    """Only the norm, only the sum, and no residual."""
    x, r, w = normal(7, 40, seed=1), normal(7, 40, seed=2), normal(40, seed=3)
    d = normal(7, 40, seed=4, grad=False)
    kr.add_rms_norm(x, w, r).sum.backward(d)
    assert torch.equal(x.grad, d) and torch.equal(r.grad, d)
    assert w.grad is None or (w.grad == 0).all()
    x.grad = r.grad = w.grad = None
    n = kr.add_rms_norm(x, w, r)
    n.out.backward(d)
    dx, dw = kr.add_rms_norm_backward(d, n.sum.detach(), w.detach(), n.rstd)
    assert torch.equal(x.grad, dx) and torch.equal(r.grad, dx)
    assert torch.equal(w.grad, dw.to(w.dtype))
    x.grad = w.grad = None
    n = kr.add_rms_norm(x, w)
    assert n.sum is x
    (n.out.float() * d.float()).sum().backward()
    dx, dw = kr.add_rms_norm_backward(d, x.detach(), w.detach(), n.rstd)
    assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw.to(w.dtype))


def test_weights_alone_and_inputs_alone(kr):
    x, r, w = normal(7, 40, seed=1), normal(7, 40, seed=2), normal(40, seed=3)
    d = normal(7, 40, seed=4, grad=False)
    kr.add_rms_norm(x.detach(), w, r.detach()).out.backward(d)
    kr.add_rms_norm(x, w.detach(), r.detach()).out.backward(d)
    n = kr.add_rms_norm(x.detach(), w.detach(), r.detach())
    dx, dw = kr.add_rms_norm_backward(d, n.sum, w.detach(), n.rstd)
    assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw.to(w.dtype)) and r.grad is None
    a, g, u = normal(40, 72, seed=5), normal(56, 72, seed=6), normal(56, 72, seed=7)
    dh = normal(40, 56, seed=8, grad=False)
    kr.gated_projection(a.detach(), g, u.detach()).backward(dh)
    _, dwg, _ = kr.gated_projection_backward(dh, a.detach(), g.detach(), u.detach())
    assert torch.equal(g.grad, dwg) and a.grad is None and u.grad is None


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_gated(kr, dtype, act):
    x = normal(3, 20, 72, seed=1, dtype=dtype)
    wg, wu = normal(56, 72, seed=2, dtype=dtype), normal(56, 72, seed=3, dtype=dtype)
    dh = normal(3, 20, 56, seed=4, dtype=dtype, grad=False)
    h = kr.gated_projection(x, wg, wu, act)
    h.backward(dh)
    want = kr.gated_projection_backward(dh, x.detach(), wg.detach(), wu.detach(), act)
    for t, g in zip((x, wg, wu), want):
        assert torch.equal(t.grad, g)
    with torch.no_grad():
        assert torch.equal(h, kr.gated_projection(x, wg, wu, act))


def test_a_step_moves_every_weight(kr):
    """Norm, projection and a mean over an expanded (stride 0) gradient, twice, on another stream
    than the default: each weight gets its gradient."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        w = normal(72, seed=1)
        wg, wu = normal(56, 72, seed=2), normal(56, 72, seed=3)
        for k in range(2):
            x, r = normal(40, 72, seed=4 + k, grad=False), normal(40, 72, seed=8 + k, grad=False)
            for p in (w, wg, wu):
                p.grad = None
            n = kr.add_rms_norm(x, w, r)
            kr.gated_projection(n.out, wg, wu).sum().backward()
            one = torch.ones(40, 56, dtype=x.dtype, device="cuda")
            with torch.no_grad():
                m = kr.add_rms_norm(x, w, r)
                dn, dwg, dwu = kr.gated_projection_backward(one, m.out, wg, wu)
                _, dw = kr.add_rms_norm_backward(dn, m.sum, w, m.rstd)
            assert torch.equal(w.grad, dw.to(w.dtype))
            assert torch.equal(wg.grad, dwg) and torch.equal(wu.grad, dwu)
    torch.cuda.current_stream().wait_stream(side)


def test_no_second_derivative(kr):
    x, wg, wu = normal(40, 72, seed=5), normal(56, 72, seed=6), normal(56, 72, seed=7)
    h = kr.gated_projection(x, wg, wu)
    g, = torch.autograd.grad(h.float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.float().sum().backward()


def test_what_has_no_gradient(kr):
    """Rounding to 8 bits: refused while a graph is recorded, taken without one."""
    x, w = normal(40, 72, seed=5), normal(72, seed=6)
    with pytest.raises(ValueError):
        kr.add_rms_norm_bytes(x, w.detach())
    with pytest.raises(ValueError):
        kr.add_rms_norm_bytes(x.detach(), w.detach(), x)
    with torch.no_grad():
        q = kr.add_rms_norm_bytes(x, w)
    b = q.q[:9].clone()
    with pytest.raises(ValueError):
        kr.byte_matmul(q.q, q.scale.clone().requires_grad_(), b, q.scale[:9])
    assert kr.byte_matmul(q.q, q.scale, b, q.scale[:9]).shape == (40, 9)
