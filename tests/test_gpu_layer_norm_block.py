"""Layer norm, dropout and the 8-bit linear layers as a block uses them: a training step through torch's
graph gives what the operators give one by one, its gradients follow the formulas, and the example
plans it."""

import ctypes

import pytest
import torch

from tests.philox import factor
from tests.scaled_form import hold, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kr():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2601_17654_amd import binding

    return binding


def normal(*shape, seed, dtype, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (size * torch.randn(*shape, generator=g)).to(dtype)


def leaves(width, hidden, dtype, tokens=(3, 50)):
    got = dict(x=normal(*tokens, width, seed=1, dtype=dtype), r=normal(*tokens, width, seed=2, dtype=dtype),
               w=1 + normal(width, seed=3, dtype=dtype, size=0.2), b=normal(width, seed=4, dtype=dtype),
               up=normal(hidden, width, seed=5, dtype=dtype, size=width ** -0.5),
               down=normal(width, hidden, seed=6, dtype=dtype, size=hidden ** -0.5))
    return {k: v.to(dtype).cuda().requires_grad_() for k, v in got.items()}


def block(kr, t, p, seed):
    n = kr.add_layer_norm(t["x"], t["w"], t["b"], t["r"], p=p, seed=seed, offset=0)
    h = torch.relu(kr.scaled_linear(n.out, t["up"]))
    return kr.dropout(kr.scaled_linear(h, t["down"]), p, seed, 1, n.sum)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_step(kr, dtype, p):
    t = leaves(200, 264, dtype)
    seed = torch.tensor([99], device="cuda")
    d = normal(3, 50, 200, seed=7, dtype=dtype).cuda()
    y = block(kr, t, p, seed)
    y.backward(d)
    # the same by the operators' own calls
    with torch.no_grad():
        n = kr.add_layer_norm(t["x"], t["w"], t["b"], t["r"], p=p, seed=99)
        u = kr.scaled_linear(n.out, t["up"])
        h = torch.relu(u)
        v = kr.scaled_linear(h, t["down"])
        assert torch.equal(y, kr.dropout(v, p, 99, 1, n.sum))
        dv = kr.dropout(d, p, 99, 1)
        dh, ddown = kr.scaled_linear_backward(dv, h, t["down"])
        dn, dup = kr.scaled_linear_backward(torch.where(u > 0, dh, torch.zeros_like(dh)), n.out, t["up"])
        dx, dr, dw, db = kr.add_layer_norm_backward(dn, n.sum, t["w"], n.mean, n.rstd, d, p, 99)
    for k, g in dict(x=dx, r=dr, w=dw.to(dtype), b=db.to(dtype), up=dup, down=ddown).items():
        assert torch.equal(t[k].grad, g), k


def test_step_against_the_formulas(kr):
    """Float32, where a value beside an 8-bit step's border is rare: the step's output and gradients in 64
    bits, values held where the operators hold them.  What 32 bits leave of a held value's border
    (about one in 2^16 of 40,000) is a step of 2^-4 of that value: against a tensor's norm below 1e-3."""
    t = leaves(200, 264, torch.float32)
    d = normal(3, 50, 200, seed=7, dtype=torch.float32)
    block(kr, t, 0.2, 99).backward(d.cuda())

    def held(v, square=False):
        return values(*hold(v, square))

    x, r, w, b, up, down = (t[k].detach().double().cpu() for k in ("x", "r", "w", "b", "up", "down"))
    x, r, d = (v.reshape(150, 200).double() for v in (x, r, d))
    f0, f1 = (factor(150, 200, 0.2, 99, o) for o in (0, 1))
    s = x * f0 + r
    c = s - s.mean(-1, keepdim=True)
    f = 1 / (c.square().mean(-1, keepdim=True) + 1e-5).sqrt()
    n = (c * f * w + b)
    u = held(n) @ held(up, True).t()
    h = u.clamp_min(0)
    dv = d * f1
    dh = held(dv) @ held(down.t(), True).t()
    ddown = held(dv.t()) @ held(h.t()).t()
    du = torch.where(u > 0, dh, torch.zeros_like(dh))
    dn = held(du) @ held(up.t(), True).t()
    dup = held(du.t()) @ held(n.t()).t()
    e, g = c * f, dn * w
    dr = f * (g - g.mean(-1, keepdim=True) - e * (g * e).mean(-1, keepdim=True)) + d
    want = dict(x=dr * f0, r=dr, w=(dn * e).sum(0), b=dn.sum(0), up=dup, down=ddown)
    for k, v in want.items():
        got = t[k].grad.double().cpu().reshape(v.shape)
        assert float((got - v).norm() / v.norm()) < 1e-3, k


def test_captured_step(kr):
    """Forward and backward through torch's graph in one captured graph, replayed with new inputs and seeds,
    beside eager steps on another stream."""
    t = {k: v.detach() for k, v in leaves(200, 264, torch.bfloat16).items()}
    d = normal(3, 50, 200, seed=7, dtype=torch.bfloat16).cuda()
    seed = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step(s):
        own = {k: v.clone().requires_grad_() for k, v in t.items()}
        y = block(kr, own, 0.2, s)
        return (y.detach(), *torch.autograd.grad(y, list(own.values()), d))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(seed)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(seed)
    for k in range(4):
        seed.fill_(5 + k)
        t["x"].copy_(normal(3, 50, 200, seed=30 + k, dtype=torch.bfloat16))
        t["up"].mul_(0.9)
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(side):
            want = step(5 + k)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
        torch.cuda.synchronize()


def test_two_streams_at_once(kr):
    """The same calls on two streams, interleaved: neither touches what the other uses."""
    t = {k: v.detach() for k, v in leaves(520, 1032, torch.bfloat16, (4, 150)).items()}
    d = normal(4, 150, 520, seed=7, dtype=torch.bfloat16).cuda()

    def step():
        own = {k: v.clone().requires_grad_() for k, v in t.items()}
        y = block(kr, own, 0.2, 3)
        return (y.detach(), *torch.autograd.grad(y, list(own.values()), d))

    want = step()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for k in range(6):
        with torch.cuda.stream(streams[k % 2]):
            got.append(step())
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_linear_to_rows_apart(kr):
    """The C calls to rows apart, each gradient alone and both: gaps and rows behind stay; without rows the
    weight's gradient is zeros."""
    L, t = kr._lib, kr._TYPES[torch.bfloat16]
    x, w = normal(70, 130, seed=1, dtype=torch.bfloat16).cuda(), normal(50, 130, seed=2, dtype=torch.bfloat16).cuda()
    d = normal(70, 50, seed=3, dtype=torch.bfloat16).cuda()
    y, (dx, dw) = kr.scaled_linear(x, w), kr.scaled_linear_backward(d, x, w)
    for rows in (70, 0):
        l = kr.KrLinear(t, rows, 130, 50, x.data_ptr(), w.data_ptr(), 130, 130)
        n = max(L.kr_scaled_linear_workspace(l), L.kr_scaled_linear_backward_workspace(l))
        ws, at = kr._scratch(n)
        out, gx, gw = (torch.full((r + 1, c + 6), 7.0, dtype=torch.bfloat16, device="cuda")
                       for r, c in ((70, 50), (70, 130), (50, 130)))
        st = kr._raw_stream(0)
        assert L.kr_scaled_linear(ctypes.byref(l), out.data_ptr(), 56, at, n, st) == kr.KR_OK
        assert (out[:rows, 50:] == 7).all() and (out[rows:] == 7).all()
        for to_x, to_w in ((gx, gw), (gx, None), (None, gw), (None, None)):
            gx.fill_(7.0)
            gw.fill_(7.0)
            assert L.kr_scaled_linear_backward(
                ctypes.byref(l), d.data_ptr(), 50, None if to_x is None else gx.data_ptr(), 136,
                None if to_w is None else gw.data_ptr(), 136, at, n, st) == kr.KR_OK
            assert (gx[rows:] == 7).all() and (gx[:, 130:] == 7).all()
            assert (gw[50] == 7).all() and (gw[:, 130:] == 7).all()
            if to_x is not None:
                assert torch.equal(gx[:rows, :130], dx[:rows])
            else:
                assert (gx == 7).all()
            if to_w is not None:
                assert torch.equal(gw[:50, :130], dw if rows else torch.zeros_like(dw))
            else:
                assert (gw == 7).all()
        if rows:
            assert torch.equal(out[:70, :50], y)


def test_the_example_plans_it(kr, capsys):
    from examples import plan_block as E

    times, r = E.run_layer_norm_block(200, 264, 130, repeats=2)
    assert set(times) == {k for p in E.LAYER_NORM for k in p}
    assert all(s > 0 and b > 0 for s, b in times.values())
    for v in (r["layer_norm"].out, r["linear"], *r["linear_back"], *r["layer_norm_back"]):
        assert torch.isfinite(v).all()
    T, E_, sched = E.main(["--block", "layer_norm", "--rows", "200", "--width", "264", "--hidden", "130",
                           "--layers", "2"])
    assert len(T) >= 1 and sched.shape == (len(T), 4, 3)
    text = capsys.readouterr().out
    assert "layer_norm + linear" in text and "linear_back + layer_norm_back" in text
