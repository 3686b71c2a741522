"""Performance cases of the transformer-block operators: the compute kernels of a training
partition (norm with the residual's addition, gated projection), their backward passes, and
the forward form in 8-bit integers.

`run` computes an operator in plain torch operations (32 bits, rounded once at the end), or,
where `own` is true, through paper_2601_17654_amd.binding.  The kinds:

  norm        sum of input and residual, its root-mean-square norm, and each row's factor
  norm_bytes  the same with the norm held in 8-bit integers and a scale per row
  norm_back   gradients of the input and of the norm's weight
  bytes       product of 8-bit integers with a scale per row of either side
  gated       act(x Wg^T) * (x Wu^T)
  gated_back  gradients of x, Wg and Wu, from the operator's inputs alone
"""

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6
TINY = 2.0 ** -100  # a row whose largest value is below this is held as zeros


def listed():
    return [
        # One token of a decoding step: latency.
        dict(name="norm_token", kind="norm", rows=1, width=4096, type="bf16"),
        # A microbatch of training tokens.
        dict(name="norm_train", kind="norm", rows=16384, width=4096, type="bf16"),
        # Its backward pass.
        dict(name="norm_back_train", kind="norm_back", rows=16384, width=4096, type="bf16"),
        # A ragged batch in 32 bits, a width that no vector load divides.
        dict(name="norm_back_ragged", kind="norm_back", rows=1531, width=2057, type="f32"),
        # The input of an 8-bit projection, a prompt's tokens.
        dict(name="norm_bytes_prompt", kind="norm_bytes", rows=8192, width=8192, type="f16"),
        # 8-bit projection of one token: the weights are read once.
        dict(name="bytes_token", kind="bytes", m=1, n=8192, k=8192, type="bf16"),
        # Sizes that are multiples of nothing.
        dict(name="bytes_ragged", kind="bytes", m=333, n=5001, k=2059, type="f32"),
        # 8-bit projection of a prompt.
        dict(name="bytes_prompt", kind="bytes", m=8192, n=8192, k=8192, type="bf16"),
        # Gated projection of one token.
        dict(name="gated_token", kind="gated", rows=1, width=4096, hidden=14336, act="silu",
             type="bf16"),
        # A training microbatch, forward.
        dict(name="gated_train", kind="gated", rows=8192, width=4096, hidden=14336, act="silu",
             type="bf16"),
        # Backward of a small ragged batch.
        dict(name="gated_back_ragged", kind="gated_back", rows=1111, width=1030, hidden=2731,
             act="gelu", type="f16"),
        # The training microbatch, backward.
        dict(name="gated_back_train", kind="gated_back", rows=8192, width=4096, hidden=14336,
             act="silu", type="bf16"),
    ]


def _size(rng, lo, hi):
    """Log-uniform size; half of them rounded to a multiple of 64, as model widths are."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and v >= 64:
        v = v // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    most = {c["name"]: work(c) for c in listed()}
    kind = rng.choice(["norm", "norm_bytes", "norm_back", "bytes", "gated", "gated_back"])
    while True:
        if kind.startswith("norm"):
            c = dict(kind=kind, rows=_size(rng, 1, 16384), width=_size(rng, 64, 16384))
            top = "norm_train"
        elif kind == "bytes":
            c = dict(kind=kind, m=_size(rng, 1, 16384), n=_size(rng, 64, 16384),
                     k=_size(rng, 64, 16384))
            top = "bytes_prompt"
        else:
            c = dict(kind=kind, rows=_size(rng, 1, 8192), width=_size(rng, 64, 8192),
                     hidden=_size(rng, 64, 16384), act=rng.choice(["silu", "gelu"]))
            top = "gated_train" if kind == "gated" else "gated_back_train"
        # 32 bits where the operator gives them back: held values are compared in 16
        c["type"] = rng.choice(["bf16", "f16", "f32"] if kind in ("norm", "norm_back", "bytes")
                               else ["bf16", "f16"])
        w = work(c)
        sizes = [v for v in c.values() if isinstance(v, int)]
        if (3072 not in sizes and w["flops"] <= most[top]["flops"]
                and w["bytes"] <= 2 * most[top]["bytes"]):
            return c


def work(case):
    b = {"bf16": 2, "f16": 2, "f32": 4}[case["type"]]
    if case["kind"] == "bytes":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k + n * k + m * n * b + 4 * (m + n), "flops": 2 * m * n * k}
    t, d = case["rows"], case["width"]
    if case["kind"] == "norm":  # x, residual, weight; sum, norm, factors
        return {"bytes": 4 * t * d * b + d * b + 4 * t, "flops": 5 * t * d}
    if case["kind"] == "norm_bytes":  # the norm in one byte, factors and scales
        return {"bytes": t * d * (3 * b + 1) + d * b + 8 * t, "flops": 7 * t * d}
    if case["kind"] == "norm_back":  # sum, two gradients, weight, factors; two gradients
        return {"bytes": 4 * t * d * b + d * (b + 4) + 4 * t, "flops": 10 * t * d}
    f = case["hidden"]
    if case["kind"] == "gated":
        return {"bytes": b * (t * d + 2 * f * d + t * f), "flops": 4 * t * d * f}
    return {"bytes": b * (2 * t * d + 4 * f * d + t * f), "flops": 12 * t * d * f}


def _inputs(case, seed):
    """The inputs alone, by name."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["type"]]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    if case["kind"] == "bytes":
        m, n, k = case["m"], case["n"], case["k"]

        def held(rows):  # rows held in 8 bits: normal values, the largest of a row at 127
            return (normal(rows, k) * 30.0).round().clamp(-127, 127).to(torch.int8)

        def scales(rows):
            return torch.exp(0.5 * normal(rows)) / 30.0

        return dict(a=held(m), sa=scales(m), b=held(n), sb=scales(n) / math.sqrt(k))
    t, d = case["rows"], case["width"]
    if case["kind"].startswith("norm"):
        # activations: tokens and channels differ in size, a few channels by much
        channel = torch.exp(0.3 * normal(d)) * (1.0 + 15.0 * (normal(d) > 2.8))
        weight = (1.0 + 0.2 * normal(d)).to(dt)
        if case["kind"] == "norm_back":
            s = (normal(t, d) * channel).to(dt)
            rstd = torch.rsqrt(s.float().square().mean(-1) + EPS)
            return dict(s=s, weight=weight, rstd=rstd, dout=normal(t, d).to(dt),
                        dsum=normal(t, d).to(dt))
        return dict(x=normal(t, d).to(dt), residual=(normal(t, d) * channel).to(dt),
                    weight=weight)
    f = case["hidden"]
    got = dict(x=normal(t, d).to(dt), wg=(normal(f, d) / math.sqrt(d)).to(dt),
               wu=(normal(f, d) / math.sqrt(d)).to(dt))
    if case["kind"] == "gated_back":
        got["dh"] = normal(t, f).to(dt)
    return got


def prepare(case, seed):
    return dict(case=case, **_inputs(case, seed))


def _act(g, name):
    """The activation and its derivative."""
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    k = math.sqrt(2.0 / math.pi)
    th = torch.tanh(k * (g + 0.044715 * g * g * g))
    return (0.5 * g * (1.0 + th),
            0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * k * (1.0 + 3 * 0.044715 * g * g))


def _run_own(state):
    from paper_2601_17654_amd import binding as kr

    case = state["case"]
    kind = case["kind"]
    if kind == "norm":
        r = kr.add_rms_norm(state["x"], state["weight"], residual=state["residual"], eps=EPS)
        return dict(sum=r.sum, out=r.out, rstd=r.rstd)
    if kind == "norm_bytes":
        r = kr.add_rms_norm_bytes(state["x"], state["weight"], residual=state["residual"], eps=EPS)
        values = torch.empty_like(state["x"])
        torch.mul(r.q, r.scale[:, None], out=values)
        return dict(sum=r.sum, values=values, scale=r.scale, rstd=r.rstd)
    if kind == "norm_back":
        dx, dw = kr.add_rms_norm_backward(state["dout"], state["s"], state["weight"],
                                          state["rstd"], dsum=state["dsum"])
        return dict(dx=dx, dweight=dw)
    if kind == "bytes":
        return kr.byte_matmul(state["a"], state["sa"], state["b"], state["sb"],
                              dtype=TYPES[case["type"]])
    if kind == "gated":
        return kr.gated_projection(state["x"], state["wg"], state["wu"], act=case["act"])
    dx, dwg, dwu = kr.gated_projection_backward(state["dh"], state["x"], state["wg"], state["wu"],
                                                act=case["act"])
    return dict(dx=dx, dwg=dwg, dwu=dwu)


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    kind, dt = case["kind"], TYPES[case["type"]]
    if kind in ("norm", "norm_bytes"):
        s = state["x"].float() + state["residual"].float()
        rstd = 1.0 / torch.sqrt((s * s).mean(-1) + EPS)
        n = s * rstd[:, None] * state["weight"].float()
        if kind == "norm":
            return dict(sum=s.to(dt), out=n.to(dt), rstd=rstd)
        top = n.abs().amax(-1)
        held = (top >= TINY) & torch.isfinite(top)
        inv = torch.where(held, 127.0 / top, torch.zeros_like(top))
        scale = torch.where(held, top / 127.0, top * 0.0)
        q = torch.where(held[:, None], torch.round(n * inv[:, None]), torch.zeros_like(n))
        return dict(sum=s.to(dt), values=(q * scale[:, None]).to(dt), scale=scale, rstd=rstd)
    if kind == "norm_back":
        h = state["s"].float() * state["rstd"][:, None]
        dout = state["dout"].float()
        dn = dout * state["weight"].float()
        c = (dn * h).mean(-1, keepdim=True)
        dx = (dn - h * c) * state["rstd"][:, None] + state["dsum"].float()
        return dict(dx=dx.to(dt), dweight=(dout * h).sum(0))
    if kind == "bytes":
        y = state["a"].float() @ state["b"].float().t()
        return (y * state["sa"][:, None] * state["sb"]).to(dt)
    x, wg, wu = state["x"].float(), state["wg"].float(), state["wu"].float()
    g, u = x @ wg.t(), x @ wu.t()
    v, slope = _act(g, case["act"])
    if kind == "gated":
        return (v * u).to(dt)
    dh = state["dh"].float()
    dg, du = dh * u * slope, dh * v
    return dict(dx=(dg @ wg + du @ wu).to(dt), dwg=(dg.t() @ x).to(dt), dwu=(du.t() @ x).to(dt))


def exact(case, seed):
    """The operator's definition in 64 bits, apart from the forms above."""
    i = {k: v.double() for k, v in _inputs(case, seed).items()}
    kind = case["kind"]
    if kind == "bytes":
        return torch.mm(i["a"] * i["sa"].unsqueeze(1), (i["b"] * i["sb"].unsqueeze(1)).t())
    if kind == "norm" or kind == "norm_bytes":
        total = torch.add(i["x"], i["residual"])
        power = torch.linalg.vector_norm(total, dim=1).square() / case["width"]
        factor = torch.pow(power + EPS, -0.5)
        normed = torch.einsum("td,t,d->td", total, factor, i["weight"])
        if kind == "norm":
            return dict(sum=total, out=normed, rstd=factor)
        largest = torch.maximum(normed.max(1).values, -normed.min(1).values)
        unit = largest / 127
        steps = torch.div(normed, unit.clamp_min(TINY / 127).unsqueeze(1)).round()
        return dict(sum=total, values=steps * unit.unsqueeze(1), scale=unit, rstd=factor)
    if kind == "norm_back":
        # the gradient of sum(dout * w * s * rstd(s)) + sum(dsum * s), rstd as it was kept
        s, w, f, d = i["s"], i["weight"], i["rstd"], i["dout"]
        along = torch.einsum("td,d,td->t", d, w, s)
        cube = f.pow(3) / case["width"] * along
        dx = torch.einsum("td,d,t->td", d, w, f) - s * cube.unsqueeze(1) + i["dsum"]
        return dict(dx=dx, dweight=torch.einsum("td,td,t->d", d, s, f))
    a, b = torch.mm(i["x"], i["wg"].t()), torch.mm(i["x"], i["wu"].t())
    with torch.enable_grad():
        a.requires_grad_(True)
        if case["act"] == "silu":
            curve = torch.sigmoid(a) * a
        else:
            curve = torch.nn.functional.gelu(a, approximate="tanh")
        slope, = torch.autograd.grad(curve.sum(), a)
    curve = curve.detach()
    if kind == "gated":
        return curve * b
    da, db = i["dh"] * b * slope, i["dh"] * curve
    return dict(dx=torch.mm(da, i["wg"]) + torch.mm(db, i["wu"]), dwg=torch.mm(da.t(), i["x"]),
                dwu=torch.mm(db.t(), i["x"]))
