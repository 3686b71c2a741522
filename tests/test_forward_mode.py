"""Forward-mode derivatives: the operators have none, and a tensor that carries a tangent is refused before
anything else is asked of it, whichever argument it is; without one, calls inside a level go on as ever."""

import pytest
import torch
import torch.autograd.forward_ad as forward

from paper_2601_17654_amd import binding as b

ROWS, WIDTH, HIDDEN = 4, 8, 6


def inputs():
    def m(*shape):
        return torch.ones(*shape)

    q = m(ROWS, WIDTH).to(torch.float8_e4m3fn)
    return dict(x=m(ROWS, WIDTH), r=m(ROWS, WIDTH), w=m(WIDTH), bias=m(WIDTH), mean=m(ROWS), rstd=m(ROWS),
                dout=m(ROWS, WIDTH), dsum=m(ROWS, WIDTH), up=m(HIDDEN, WIDTH), up2=m(HIDDEN, WIDTH),
                dh=m(ROWS, HIDDEN), sa=m(ROWS), sb=m(HIDDEN), qa=q, qb=q.clone())


def held(q):
    return b.Scaled(q, torch.zeros(1, 128, dtype=torch.uint8))


BYTES = torch.zeros(ROWS, WIDTH, dtype=torch.int8), torch.zeros(HIDDEN, WIDTH, dtype=torch.int8)
CALLS = {
    "dropout": (lambda t: b.dropout(t["x"], 0.1, 0, 0, t["r"]), "x r"),
    "add_rms_norm": (lambda t: b.add_rms_norm(t["x"], t["w"], t["r"]), "x w r"),
    "add_rms_norm_bytes": (lambda t: b.add_rms_norm_bytes(t["x"], t["w"], t["r"]), "x w r"),
    "add_rms_norm_backward": (
        lambda t: b.add_rms_norm_backward(t["dout"], t["x"], t["w"], t["rstd"], t["dsum"]),
        "dout x w rstd dsum"),
    "add_layer_norm": (lambda t: b.add_layer_norm(t["x"], t["w"], t["bias"], t["r"], p=0.1), "x w bias r"),
    "add_layer_norm_backward": (
        lambda t: b.add_layer_norm_backward(t["dout"], t["x"], t["w"], t["mean"], t["rstd"], t["dsum"]),
        "dout x w mean rstd dsum"),
    "gated_projection": (lambda t: b.gated_projection(t["x"], t["up"], t["up2"]), "x up up2"),
    "gated_projection_backward": (
        lambda t: b.gated_projection_backward(t["dh"], t["x"], t["up"], t["up2"]), "dh x up up2"),
    "byte_matmul": (lambda t: b.byte_matmul(BYTES[0], t["sa"], BYTES[1], t["sb"]), "sa sb"),
    "scaled_hold": (lambda t: b.scaled_hold(t["x"]), "x"),
    "scaled_values": (lambda t: b.scaled_values(held(t["qa"])), "qa"),
    "scaled_matmul": (lambda t: b.scaled_matmul(held(t["qa"]), held(t["qb"])), "qa qb"),
    "scaled_linear": (lambda t: b.scaled_linear(t["x"], t["up"]), "x up"),
    "scaled_linear of a held weight": (lambda t: b.scaled_linear(t["x"], held(t["qb"])), "x qb"),
    "scaled_linear_backward": (lambda t: b.scaled_linear_backward(t["dh"], t["x"], t["up"]), "dh x up"),
}


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("call,name", [(c, n) for c, (_, names) in CALLS.items() for n in names.split()])
def test_refused(call, name, graph):
    with forward.dual_level(), torch.set_grad_enabled(graph):
        t = inputs()
        t[name] = forward.make_dual(t[name], torch.ones_like(t[name]))
        with pytest.raises(ValueError, match="forward-mode"):
            CALLS[call][0](t)
        if graph and call + "_backward" in CALLS:  # what takes part in a graph too
            t["x" if name != "x" else list(t)[2]].requires_grad_()
            with pytest.raises(ValueError, match="forward-mode"):
                CALLS[call][0](t)


@pytest.mark.parametrize("call", CALLS)
def test_without_tangents(call):
    """The next thing is said, here that the tensors are not on the device or of another type."""
    with forward.dual_level():
        with pytest.raises((ValueError, TypeError)) as said:
            CALLS[call][0](inputs())
        assert "forward-mode" not in str(said.value)
