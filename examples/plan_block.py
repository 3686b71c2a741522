"""Plan a transformer block from kernel times measured on this card.

Runs the compute kernels of a block's feed-forward half -- forward (norm with the residual's
addition, gated projection), backward (their gradients) and the forward form in 8-bit integers
(norm held in bytes, byte product) -- times each, expands the times to the planner's tables and
plans two steps: training (forward and backward) and a forward step in 8 bits.  For either it
prints the time-energy frontier's size and the schedule of its fastest and its cheapest point.

    python examples/plan_block.py [--rows 8192] [--width 4096] [--hidden 14336] [--layers 16]

What is measured is each kernel's time with all compute units at the clock of the moment.  How a
time changes with frequency and with units given to communication is the table generator's
formula: a kernel's share alpha that scales with the clock, and its exponent beta in the units,
are set from how its operations compare with its bytes.  Powers and the communication's bandwidth
are the generator's, too.
"""

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_17654_amd import binding as kr  # noqa: E402
from paper_2601_17654_amd import inputs as I  # noqa: E402

UNITS = 256.0                # compute units
BALANCE = 250.0              # operations per byte where the two cost the same (16 bits)


def measure(fn, repeats=10):
    """Median time of fn in seconds, and its last result."""
    out = fn()
    times = []
    for _ in range(repeats):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        out = fn()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b) * 1e-3)
    return float(np.median(times)), out


def held(w):
    """A weight matrix in 8-bit integers with a scale for each row."""
    scale = w.float().abs().amax(1) / 127.0
    return torch.round(w.float() / scale[:, None]).to(torch.int8), scale


def run_block(rows, width, hidden, repeats=10):
    """One pass of every kernel, in order of use: {name: (seconds, operations per byte)}, and the
    results, by name."""
    gen = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)

    x, residual, dh, dsum = (normal(rows, width), normal(rows, width), normal(rows, hidden),
                             normal(rows, width))
    weight = torch.ones(width, dtype=torch.bfloat16, device="cuda")
    wg, wu = normal(hidden, width) / width ** 0.5, normal(hidden, width) / width ** 0.5
    b, sb = held(wg)
    t, r = {}, {}
    t["norm"], r["norm"] = measure(lambda: kr.add_rms_norm(x, weight, residual), repeats)
    n = r["norm"]
    t["gated"], r["gated"] = measure(lambda: kr.gated_projection(n.out, wg, wu), repeats)
    t["gated_back"], r["gated_back"] = measure(
        lambda: kr.gated_projection_backward(dh, n.out, wg, wu), repeats)
    dn = r["gated_back"][0]
    t["norm_back"], r["norm_back"] = measure(
        lambda: kr.add_rms_norm_backward(dn, n.sum, weight, n.rstd, dsum), repeats)
    t["norm_bytes"], r["norm_bytes"] = measure(
        lambda: kr.add_rms_norm_bytes(x, weight, residual), repeats)
    q = r["norm_bytes"]
    t["bytes"], r["bytes"] = measure(lambda: kr.byte_matmul(q.q, q.scale, b, sb), repeats)
    mw, wh, mh = rows * width, width * hidden, rows * hidden
    per_byte = {"norm": 5 * mw / (8.0 * mw), "norm_back": 10 * mw / (8.0 * mw),
                "norm_bytes": 7 * mw / (7.0 * mw),
                "gated": 4.0 * mw * hidden / (2 * (mw + 2 * wh + mh)),
                "gated_back": 12.0 * mw * hidden / (2 * (2 * mw + 4 * wh + mh)),
                "bytes": mw * hidden / (1.0 * mw + wh + 2 * mh)}  # 8 bits: half the cost each
    return {k: (t[k], per_byte[k]) for k in t}, r


# The block's partitions: kernels that run beside one collective each.
PARTITIONS = (("norm", "gated"), ("gated_back", "norm_back"), ("norm_bytes", "bytes"))
TRAINING, BYTES_FORWARD = PARTITIONS[:2], PARTITIONS[2:]  # those of one step


def tables(times, layers, rows, width, partitions=PARTITIONS):
    """The planner's space and tables of `layers` blocks of such partitions."""
    space = I.Space(n_parts=len(partitions) * layers, n_kernels=2, n_comm=1, n_pos=3,
                    sm_counts=tuple(range(8, 65, 8)), total_sms=UNITS,
                    freqs_mhz=tuple(float(x) for x in np.linspace(1200.0, 2400.0, 25)))
    t0, per_byte = np.array([[times[k] for k in p] for p in partitions] * layers).transpose(2, 0, 1)
    share = per_byte / (per_byte + BALANCE)   # of the cost that is operations
    P, N = t0.shape
    ones = np.ones((P, N))
    return space, I.expand_tables(space, t0, 0.3 + 0.7 * share, 0.2 + 0.8 * share,
                                  300.0 + 400.0 * share, 2.0 * ones,
                                  np.full((P, 1), 2.0 * rows * width), np.full((P, 1), 140.0))


def plan(space, tabs, bins=8192):
    """The step's frontier: (times, energies, schedules [points][partitions] as (frequency index,
    launch position, unit choice))."""
    dev = [torch.from_numpy(tabs[k]).cuda() for k in ("t", "pw", "tc", "pc")]
    fr = kr.evaluate_and_filter(space, *dev)
    comp = kr.compose_frontiers(fr.off, fr.T, fr.E, bins)
    stair, _, _ = comp.staircase()
    _, cand, T, E, ok = kr.extract_schedule(comp, fr.off, fr.T, fr.E, stair, cand_idx=fr.idx)
    assert bool(ok.all())
    # composed on a grid of time bins: the exact sums of neighbouring bins may change places
    best = kr.pareto_filter(T, E, [0, T.numel()])
    cand = cand[best.idx.long()]
    f, pos, sm = kr.decode_candidates(space, cand.reshape(-1))
    shape = tuple(cand.shape)
    return (best.T.cpu().numpy(), best.E.cpu().numpy(),
            np.stack([v.cpu().numpy().reshape(shape) for v in (f, pos, sm)], axis=-1))


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--rows", type=int, default=8192)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=14336)
    ap.add_argument("--layers", type=int, default=16)
    a = ap.parse_args(argv)
    times, _ = run_block(a.rows, a.width, a.hidden)
    for name, (s, per_byte) in times.items():
        print("%-11s %9.1f us   %7.1f operations a byte" % (name, s * 1e6, per_byte))
    plans = []
    for name, partitions in (("training step", TRAINING), ("forward step in 8 bits", BYTES_FORWARD)):
        space, tabs = tables(times, a.layers, a.rows, a.width, partitions)
        T, E, sched = plan(space, tabs)
        plans.append((T, E, sched))
        print("%s: %d frontier points" % (name, len(T)))
        for what, i in (("fastest", int(np.argmin(T))), ("cheapest", int(np.argmin(E)))):
            print("%-8s %.3f ms  %.3f J" % (what, T[i] * 1e3, E[i]))
            for p, kernels in enumerate(partitions):
                f, pos, sm = sched[i, p]
                print("   %-24s %4.0f MHz, %2d units to the collective, launched %s"
                      % (" + ".join(kernels), space.freqs_mhz[f], space.sm_counts[sm],
                         "after both" if pos == 2 else "with " + kernels[pos]))
    return plans[0]


if __name__ == "__main__":
    main()
