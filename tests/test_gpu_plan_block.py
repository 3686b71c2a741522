"""The block's operators run together and planned from their times: the example's results against
64 bits, its frontier against the oracle on the same tables."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_block_is_run_and_planned(oracle_lib):
    from examples import plan_block as E

    rows, width, hidden, layers = 200, 264, 130, 3
    times, r = E.run_block(rows, width, hidden, repeats=2)
    assert set(times) == {k for p in E.PARTITIONS for k in p}
    assert all(s > 0 and b > 0 for s, b in times.values())
    for v in (r["norm"].out, r["gated"], r["gated_back"][0], r["norm_back"][0], r["bytes"]):
        assert torch.isfinite(v).all()
    assert r["gated"].shape == (rows, hidden) and r["norm_back"][0].shape == (rows, width)
    # 8-bit form of the same projection: half a step of either side's largest value a term
    full = r["norm"].out.double()
    q = r["norm_bytes"]
    held = q.q.double() * q.scale.double()[:, None]
    # the norm is rounded to bfloat16 (2^-8), the held one to half a step
    assert ((held - full).abs() <= 0.501 * q.scale.double()[:, None] + 2.0 ** -8 * full.abs()).all()

    space, tabs = E.tables(times, layers, rows, width)
    T, En, sched = E.plan(space, tabs, bins=1024)
    assert np.all(np.diff(T) > 0) and np.all(np.diff(En) < 0)
    ref = oracle_lib.evaluate_and_filter(space, *(tabs[k] for k in ("t", "pw", "tc", "pc")))
    off = np.concatenate([[0], np.cumsum([len(x[0]) for x in ref])]).astype(np.int64)
    rT, rE = np.concatenate([x[1] for x in ref]), np.concatenate([x[2] for x in ref])
    comp = oracle_lib.compose(off, rT, rE, 1024)
    stair, _, _ = oracle_lib.staircase(comp.F, comp.delta, comp.tmin_sum)
    ex = [oracle_lib.extract(off, rT, rE, comp, int(b)) for b in stair]
    keep = oracle_lib.pareto(np.array([x[1] for x in ex]), np.array([x[2] for x in ex]))
    assert len(keep) == len(T) and sched.shape[:2] == (len(T), 3 * layers)
    for i, k in enumerate(keep):
        choice, t, e = ex[int(k)]
        np.testing.assert_allclose([T[i], En[i]], [t, e], rtol=1e-9, atol=0)
        for p, c in enumerate(choice):
            f, pos, sm = (int(v) for v in sched[i, p])
            assert (f * space.n_pos + pos) * space.n_sm + sm == ref[p][0][c]
