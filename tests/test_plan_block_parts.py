"""What the example plans: a training step holds the forward and backward kernels once each, the
8-bit form is a forward step of its own."""

import numpy as np
import pytest


@pytest.fixture
def planned(monkeypatch):
    from examples import plan_block as E

    names = [k for p in E.PARTITIONS for k in p]
    times = {k: (1e-5 * (i + 1), 10.0 * (i + 1)) for i, k in enumerate(names)}
    seen = []

    def plan(space, tabs, bins=8192):
        seen.append((space, tabs))
        sched = np.zeros((2, space.n_parts, 3), dtype=np.int64)
        return np.array([1.0, 2.0]), np.array([2.0, 1.0]), sched

    monkeypatch.setattr(E, "run_block", lambda *a, **k: (times, {}))
    monkeypatch.setattr(E, "plan", plan)
    got = E.main(["--layers", "3"])
    return E, times, seen, got


def test_each_step_runs_its_kernels_once(planned):
    E, times, seen, got = planned
    assert [s.n_parts for s, _ in seen] == [3 * 2, 3 * 1]
    full = E.tables(times, 1, 8192, 4096)[1]["t"]
    for (_, tabs), parts in zip(seen, (E.TRAINING, E.BYTES_FORWARD)):
        at = [E.PARTITIONS.index(p) for p in parts] * 3
        np.testing.assert_array_equal(tabs["t"], full[at])
    assert sorted(k for p in E.TRAINING for k in p) == ["gated", "gated_back", "norm", "norm_back"]
    assert [k for p in E.BYTES_FORWARD for k in p] == ["norm_bytes", "bytes"]
    assert got[2].shape == (2, 6, 3)  # the training step's schedule


def test_output_names_each_step(planned, capsys):
    E, times, _, _ = planned
    E.main(["--layers", "1"])
    text = capsys.readouterr().out
    first, second = text.split("forward step in 8 bits")
    assert "training step" in first and "gated_back + norm_back" in first
    assert "norm_bytes + bytes" not in first and "norm_bytes + bytes" in second
    assert "norm + gated" not in second
