"""Performance cases of further transformer-block operators: layer norm with the residual's
addition and dropout, dropout alone, and products in 8-bit floating point (e4m3) with a power of
two as the scale of each 128 values along the sum.

`run` computes an operator in plain torch operations (32 bits, rounded once at the end), or,
where `own` is true, through paper_2601_17654_amd.binding.  The kinds:

  norm         s = residual + dropout(x); its layer norm, and each row's mean and factor
  norm_back    gradients of x, the residual, the norm's weight and its bias
  dropout      the kept values times 1 / (1 - p), the others 0
  hold         values held in 8 bits, with a scale for each row's (or square's) 128: as they are, for
               a sum over columns, and crossed, for a sum over rows; returned as the values held
  product      a b^T of held values
  linear       x w^T: both held (x by rows, w by squares), then their product
  linear_back  gradients of x and w, all operands held along the sum that they enter

Dropout's random numbers: value (i, c) has 16 bits, number c % 8 of the Philox4x32-10 words of
counter (c // 8, i, offset), key seed; it is kept where they are round(65536 p) or more.
"""

import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-5
B = 128      # values that share a scale
MOST = 448   # largest value of e4m3


def listed():
    return [
        # One token's norm: latency.
        dict(name="norm_token", kind="norm", rows=1, width=4096, p=0.0, type="bf16"),
        # A microbatch of training tokens, the branch dropped out.
        dict(name="norm_train", kind="norm", rows=16384, width=4096, p=0.1, type="bf16"),
        # Its backward pass.
        dict(name="norm_back_train", kind="norm_back", rows=16384, width=4096, p=0.1, type="bf16"),
        # A small batch of a width that no vector load divides.
        dict(name="dropout_ragged", kind="dropout", rows=777, width=2059, p=0.25, type="f32"),
        # A microbatch's hidden values.
        dict(name="dropout_train", kind="dropout", rows=8192, width=14336, p=0.1, type="bf16"),
        # Activations of an odd batch.
        dict(name="hold_ragged", kind="hold", rows=1531, width=2057, square=False, plain=True,
             crossed=False, type="f16"),
        # A weight for its product and for the gradient's.
        dict(name="hold_weight", kind="hold", rows=14336, width=4096, square=True, plain=True,
             crossed=True, type="bf16"),
        # One token: the weight is read once.
        dict(name="product_token", kind="product", m=1, n=8192, k=8192, type="bf16"),
        # Sizes that are multiples of nothing.
        dict(name="product_ragged", kind="product", m=333, n=5001, k=2059, type="f32"),
        # A prompt's tokens.
        dict(name="product_prompt", kind="product", m=8192, n=8192, k=8192, type="bf16"),
        # A training microbatch from 16-bit values, forward.
        dict(name="linear_train", kind="linear", rows=8192, width=4096, hidden=14336, type="bf16"),
        # And backward.
        dict(name="linear_back_train", kind="linear_back", rows=8192, width=4096, hidden=14336,
             type="bf16"),
    ]


def _size(rng, lo, hi):
    """Log-uniform size; half of them rounded to a multiple of 64, as model widths are."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and v >= 64:
        v = v // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    most = {c["name"]: work(c) for c in listed()}
    kind = rng.choice(["norm", "norm_back", "dropout", "hold", "product", "linear", "linear_back"])
    top = {"norm": "norm_train", "norm_back": "norm_back_train", "dropout": "dropout_train",
           "hold": "hold_weight", "product": "product_prompt", "linear": "linear_train",
           "linear_back": "linear_back_train"}[kind]
    while True:
        if kind == "product":
            c = dict(kind=kind, m=_size(rng, 1, 16384), n=_size(rng, 64, 16384),
                     k=_size(rng, 64, 16384))
        elif kind.startswith("linear"):
            c = dict(kind=kind, rows=_size(rng, 1, 8192), width=_size(rng, 64, 8192),
                     hidden=_size(rng, 64, 16384))
        else:
            c = dict(kind=kind, rows=_size(rng, 1, 16384), width=_size(rng, 64, 16384))
            if kind == "hold":
                c["square"] = rng.random() < 0.5
                c["plain"], c["crossed"] = rng.choice([(True, False), (False, True), (True, True)])
            else:
                c["p"] = round(rng.uniform(0.02, 0.5), 3)
                if kind != "dropout" and rng.random() < 0.5:
                    c["p"] = 0.0
        c["type"] = rng.choice(["bf16", "f16"] if kind.startswith("linear")
                               else ["bf16", "f16", "f32"])
        w = work(c)
        if w["flops"] <= most[top]["flops"] and w["bytes"] <= 2 * most[top]["bytes"]:
            return c


def work(case):
    b = {"bf16": 2, "f16": 2, "f32": 4}[case["type"]]
    kind = case["kind"]
    if kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        blocks = -(-k // B)
        return {"bytes": (m + n) * (k + blocks) + m * n * b, "flops": 2 * m * n * k}
    t, d = case["rows"], case["width"]
    if kind == "norm":  # x, residual, weight, bias; sum, norm, means, factors
        return {"bytes": 4 * t * d * b + 2 * d * b + 8 * t, "flops": 8 * t * d}
    if kind == "norm_back":  # sum, two gradients, weight, means, factors; two gradients (one, p = 0)
        outs = 2 if case["p"] else 1
        return {"bytes": (3 + outs) * t * d * b + d * (b + 8) + 8 * t, "flops": 14 * t * d}
    if kind == "dropout":
        return {"bytes": 2 * t * d * b, "flops": 2 * t * d}
    if kind == "hold":  # x; what it is held as, and its values
        forms = case["plain"] + case["crossed"]
        return {"bytes": t * d * (b + forms * (1 + b)), "flops": 3 * t * d * forms}
    f = case["hidden"]
    if kind == "linear":
        return {"bytes": b * (t * d + f * d + t * f), "flops": 2 * t * d * f}
    return {"bytes": b * (2 * t * d + 2 * f * d + t * f), "flops": 4 * t * d * f}


def _held_inputs(values):
    """Values as a program has them that held them before: 8-bit values in rows of a multiple of 16
    with zeros at their ends, exponents [rows][blocks], and those in the product's order: bytes
    [block][row], the rows of each 128 as 16 groups of row % 16."""
    rows, k = values.shape
    q, e = _held(values, False)
    store = torch.zeros(rows, -(-k // 16) * 16, dtype=torch.float8_e4m3fn, device=values.device)
    store[:, :k] = q.to(torch.float8_e4m3fn)
    byte = (e + 127).to(torch.uint8)
    blocks, groups = e.shape[1], -(-rows // B)
    order = torch.zeros(groups * B, blocks, dtype=torch.uint8, device=values.device)
    order[:rows] = byte
    order = order.view(groups, 8, 16, blocks).permute(3, 0, 2, 1).reshape(blocks, groups * B)
    return store[:, :k], e, order.contiguous(), store.shape[1]


def _inputs(case, seed):
    """The inputs alone, by name."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["type"]]
    numbers = random.Random(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def channels(d):  # channels differ in size, a few by much
        return torch.exp(0.3 * normal(d)) * (1.0 + 15.0 * (normal(d) > 2.8))

    kind = case["kind"]
    if kind == "product":
        k = case["k"]
        a, ea, oa, ra = _held_inputs(normal(case["m"], k) * channels(k))
        b, eb, ob, rb = _held_inputs(normal(case["n"], k) / math.sqrt(k))
        return dict(a=a, ea=ea, oa=oa, ra=ra, b=b, eb=eb, ob=ob, rb=rb)
    t, d = case["rows"], case["width"]
    drop = dict(seed=numbers.getrandbits(63), offset=numbers.getrandbits(40))
    if kind == "dropout":
        return dict(x=normal(t, d).to(dt), **drop)
    if kind == "hold":
        x = normal(t, d) * channels(d)
        return dict(x=x.to(dt))
    if kind.startswith("norm"):
        weight, bias = (1.0 + 0.2 * normal(d)).to(dt), (0.2 * normal(d)).to(dt)
        size = channels(d)
        if kind == "norm_back":
            s = (normal(t, d) * size + 0.1).to(dt)
            mean = s.double().mean(-1)
            rstd = torch.rsqrt((s.double() - mean[:, None]).square().mean(-1) + EPS)
            return dict(s=s, weight=weight, mean=mean.float(), rstd=rstd.float(),
                        dout=normal(t, d).to(dt), dsum=normal(t, d).to(dt), **drop)
        return dict(x=normal(t, d).to(dt), residual=(normal(t, d) * size + 0.1).to(dt),
                    weight=weight, bias=bias, **drop)
    f = case["hidden"]
    got = dict(x=(normal(t, d) * channels(d)).to(dt), w=(normal(f, d) / math.sqrt(d)).to(dt))
    if kind == "linear_back":
        got["dout"] = (normal(t, f) * channels(f)).to(dt)
    return got


def prepare(case, seed):
    return dict(case=case, **_inputs(case, seed))


# ---- the plain form --------------------------------------------------------------------

def _kept(rows, width, p, seed, offset, device):
    """(which values are kept, the factor of those)."""
    low = 0xFFFFFFFF
    groups = -(-width // 8)
    c0 = torch.arange(groups, device=device).expand(rows, groups)
    c1 = torch.arange(rows, device=device)[:, None].expand(rows, groups)
    c2, c3 = torch.full_like(c0, offset & low), torch.full_like(c0, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # 64-bit products: their bits, whatever the sign
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], dim=-1)
    halves = torch.stack([words & 0xFFFF, words >> 16], dim=-1).reshape(rows, groups * 8)
    cut = int(round(p * 65536))
    return halves[:, :width] >= cut, 65536.0 / (65536 - cut)


def _dropped(x, p, seed, offset):
    if p == 0.0:
        return x
    kept, factor = _kept(x.shape[0], x.shape[1], p, seed, offset, x.device)
    return torch.where(kept, x * factor, torch.zeros_like(x))


def _power(e):
    """2^e in 32 bits, -126 <= e <= 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _held(x, square):
    """(values of e4m3 in 32 bits, exponents of the scales, [rows][blocks])."""
    rows, k = x.shape
    blocks, tall = -(-k // B), -(-rows // B)
    high = rows if not square else tall * B
    room = torch.zeros(high, blocks * B, device=x.device)
    room[:rows, :k] = x.float()
    if square:
        top = room.view(tall, B, blocks, B).abs().amax((1, 3)).repeat_interleave(B, 0)[:rows]
    else:
        top = room.view(rows, blocks, B).abs().amax(-1)
    part, e = torch.frexp(top)
    e = torch.where(top > 0, e.to(torch.int64) - 9 + (part > 0.875), -127).clamp_min(-127)
    q = room.view(high, blocks, B)[:rows] * _power(-e)[:, :, None]
    q = q.reshape(rows, blocks * B)[:, :k].to(torch.float8_e4m3fn).float()
    return q, e


def _times(q, e):
    """Values that q and its exponents stand for, in 32 bits."""
    rows, k = q.shape
    return q * _power(e).repeat_interleave(B, 1)[:, :k]


def _values(x, square=False):
    return _times(*_held(x, square))


def _run_own(state):
    from paper_2601_17654_amd import binding as kr

    case = state["case"]
    kind = case["kind"]
    if kind == "norm":
        r = kr.add_layer_norm(state["x"], state["weight"], state["bias"],
                              residual=state["residual"], eps=EPS, p=case["p"],
                              seed=state["seed"], offset=state["offset"])
        return dict(sum=r.sum, out=r.out, mean=r.mean, rstd=r.rstd)
    if kind == "norm_back":
        dx, dres, dw, db = kr.add_layer_norm_backward(
            state["dout"], state["s"], state["weight"], state["mean"], state["rstd"],
            dsum=state["dsum"], p=case["p"], seed=state["seed"], offset=state["offset"])
        return dict(dx=dx, dresidual=dres, dweight=dw, dbias=db)
    if kind == "dropout":
        return kr.dropout(state["x"], case["p"], state["seed"], offset=state["offset"])
    if kind == "hold":
        dt = TYPES[case["type"]]
        h = kr.scaled_hold(state["x"], square=case["square"], plain=case["plain"],
                           crossed=case["crossed"])
        return [kr.scaled_values(x, dt) for x in h if x is not None]
    if kind == "product":
        return kr.scaled_matmul(kr.Scaled(state["a"], state["oa"], state["ra"]),
                                kr.Scaled(state["b"], state["ob"], state["rb"]),
                                dtype=TYPES[case["type"]])
    if kind == "linear":
        return kr.scaled_linear(state["x"], state["w"])
    dx, dw = kr.scaled_linear_backward(state["dout"], state["x"], state["w"])
    return dict(dx=dx, dw=dw)


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    kind, dt = case["kind"], TYPES[case["type"]]
    if kind == "norm":
        s = state["residual"].float() + _dropped(state["x"].float(), case["p"], state["seed"],
                                                 state["offset"])
        mean = s.mean(-1)
        away = s - mean[:, None]
        rstd = 1.0 / torch.sqrt((away * away).mean(-1) + EPS)
        n = away * rstd[:, None] * state["weight"].float() + state["bias"].float()
        return dict(sum=s.to(dt), out=n.to(dt), mean=mean, rstd=rstd)
    if kind == "norm_back":
        h = (state["s"].float() - state["mean"][:, None]) * state["rstd"][:, None]
        dout = state["dout"].float()
        g = dout * state["weight"].float()
        c = (g * h).mean(-1, keepdim=True)
        ds = (g - g.mean(-1, keepdim=True) - h * c) * state["rstd"][:, None]
        ds = ds + state["dsum"].float()
        dx = _dropped(ds, case["p"], state["seed"], state["offset"])
        return dict(dx=dx.to(dt), dresidual=ds.to(dt), dweight=(dout * h).sum(0),
                    dbias=dout.sum(0))
    if kind == "dropout":
        return _dropped(state["x"].float(), case["p"], state["seed"], state["offset"]).to(dt)
    if kind == "hold":
        got = []
        if case["plain"]:
            got.append(_values(state["x"], case["square"]).to(dt))
        if case["crossed"]:
            got.append(_values(state["x"].t(), case["square"]).to(dt))
        return got
    if kind == "product":
        a, b = _times(state["a"].float(), state["ea"]), _times(state["b"].float(), state["eb"])
        return (a @ b.t()).to(dt)
    if kind == "linear":
        return (_values(state["x"]) @ _values(state["w"], True).t()).to(dt)
    dx = _values(state["dout"]) @ _values(state["w"].t(), True).t()
    dw = _values(state["dout"].t()) @ _values(state["x"].t()).t()
    return dict(dx=dx.to(dt), dw=dw.to(dt))


# ---- the definition in 64 bits -----------------------------------------------------------

def _product_words(a, b):
    """High and low word of the product of a word with a constant, by halves."""
    a0, a1, b0, b1 = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
    middle = a1 * b0 + ((a0 * b0) >> 16)
    side = a0 * b1 + (middle & 0xFFFF)
    return a1 * b1 + (middle >> 16) + (side >> 16), (side % 65536) * 65536 + (a0 * b0) % 65536


def _exact_factor(case, i):
    """What dropout multiplies each value by."""
    rows, width = case["rows"], case["width"]
    if case["p"] == 0.0:
        return 1.0
    place = torch.arange(rows * -(-width // 8), device="cuda")
    word = [place % -(-width // 8), place // -(-width // 8),
            torch.zeros_like(place) + i["offset"] % 2 ** 32,
            torch.zeros_like(place) + i["offset"] // 2 ** 32]
    for turn in range(10):
        key = [(k + turn * step) % 2 ** 32 for k, step in
               ((i["seed"] % 2 ** 32, 0x9E3779B9), (i["seed"] // 2 ** 32, 0xBB67AE85))]
        high0, low0 = _product_words(word[0], 0xD2511F53)
        high2, low2 = _product_words(word[2], 0xCD9E8D57)
        word = [high2 ^ word[1] ^ key[0], low2, high0 ^ word[3] ^ key[1], low0]
    draws = torch.stack([w // shift % 65536 for w in word for shift in (1, 65536)], 1)
    draws = draws.reshape(rows, -1)[:, :width]
    cut = round(case["p"] * 65536)
    return (draws >= cut).double() * (65536 / (65536 - cut))


def _two(e):
    """2^e in 64 bits, of whole e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _e4m3(v):
    """The nearest value of e4m3, ties to even, of |v| <= 448."""
    octave = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6)))
    step = _two(octave - 3)
    return torch.round(v / step) * step


def _exact_held(x, square):
    rows, k = x.shape
    x = x.double()
    room = torch.nn.functional.pad(x, (0, -k % B, 0, -rows % B))
    tiles = room.unflatten(1, (-1, B)).unflatten(0, (-1, B))  # [tall][128][blocks][128]
    top = tiles.abs().amax(3, keepdim=True)
    if square:
        top = top.amax(1, keepdim=True)
    # the least e >= -127 of top <= 448 * 2^e, from one that is below it by one or two
    e = (torch.floor(torch.log2(top.clamp_min(2.0 ** -140) / MOST)) - 1).clamp_min(-127)
    unit = _two(e)
    unit = unit * (1 + (top > MOST * unit).double())
    unit = unit * (1 + (top > MOST * unit).double())
    unit = unit * (1 + (top > MOST * unit).double())
    return (_e4m3(tiles / unit) * unit).reshape(room.shape)[:rows, :k]


def exact(case, seed):
    """The operator's definition in 64 bits, apart from the forms above."""
    i = _inputs(case, seed)
    kind = case["kind"]
    if kind == "product":
        def whole(q, e):
            unit = torch.pow(2.0, e.double()).unsqueeze(2)
            room = torch.nn.functional.pad(q.double(), (0, -q.shape[1] % B))
            return (room.unflatten(1, (-1, B)) * unit).flatten(1)[:, :q.shape[1]]

        return torch.mm(whole(i["a"], i["ea"]), whole(i["b"], i["eb"]).t())
    if kind == "hold":
        return [_exact_held(v, case["square"]) for v, there in
                ((i["x"], case["plain"]), (i["x"].t(), case["crossed"])) if there]
    if kind == "linear":
        return torch.mm(_exact_held(i["x"], False), _exact_held(i["w"], True).t())
    if kind == "linear_back":
        return dict(dx=torch.mm(_exact_held(i["dout"], False), _exact_held(i["w"], True)),
                    dw=torch.mm(_exact_held(i["dout"].t(), False),
                                _exact_held(i["x"].t(), False).t()))
    factor = _exact_factor(case, i)
    if kind == "dropout":
        return i["x"].double() * factor
    if kind == "norm":
        total = torch.addcmul(i["residual"].double(), i["x"].double(),
                              torch.as_tensor(factor, dtype=torch.float64, device="cuda"))
        var, mean = torch.var_mean(total, dim=1, correction=0)
        scale = torch.pow(var + EPS, -0.5)
        normed = torch.einsum("td,t,d->td", total - mean.unsqueeze(1), scale, i["weight"].double())
        return dict(sum=total, out=normed + i["bias"].double(), mean=mean, rstd=scale)
    # the gradient of sum(dout * norm) + sum(dsum * s), means and factors as they were kept
    s, w, f, d = i["s"].double(), i["weight"].double(), i["rstd"].double(), i["dout"].double()
    away = (s - i["mean"].double().unsqueeze(1)) * f.unsqueeze(1)
    along = torch.einsum("td,d,td->t", d, w, away) / case["width"]
    level = torch.mv(d, w) / case["width"]
    ds = torch.einsum("td,d,t->td", d, w, f) - (level * f).unsqueeze(1)
    ds = ds - away * (along * f).unsqueeze(1) + i["dsum"].double()
    return dict(dx=ds * factor, dresidual=ds, dweight=torch.einsum("td,td->d", d, away),
                dbias=d.sum(0))
