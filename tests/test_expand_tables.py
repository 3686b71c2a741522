"""Tables expanded from given figures: each entry against the formula, one at a time.  Every entry
is a few products and one power in 64 bits on either side: 1e-14 relative covers them."""

import numpy as np

from paper_2601_17654_amd import inputs as I


def test_entries_follow_the_formulas():
    rng = np.random.default_rng(3)
    space = I.Space(3, 4, 2, 5, (4, 16, 24), (1000.0, 1500.0, 2000.0), total_sms=256.0)
    P, N, M = 3, 4, 2
    t0, alpha, beta = rng.uniform(1e-5, 1e-3, (P, N)), rng.uniform(0, 1, (P, N)), rng.uniform(0, 1, (P, N))
    p0, gamma = rng.uniform(300, 700, (P, N)), rng.uniform(1.5, 2.5, (P, N))
    nbytes, cpow = rng.uniform(1e6, 1e8, (P, M)), rng.uniform(80, 200, (P, M))
    t = I.expand_tables(space, t0, alpha, beta, p0, gamma, nbytes, cpow)
    avail = [256.0] + [256.0 - k for k in space.sm_counts]
    for p in range(P):
        for fi, f in enumerate(space.freqs_mhz):
            for i in range(N):
                for s, k in enumerate(avail):
                    want = t0[p, i] * (alpha[p, i] * 2000.0 / f + 1 - alpha[p, i]) * (256.0 / k) ** beta[p, i]
                    assert abs(t["t"][p, fi, i, s] / want - 1) < 1e-14
                    want = p0[p, i] * (f / 2000.0) ** gamma[p, i] * k / 256.0
                    assert abs(t["pw"][p, fi, i, s] / want - 1) < 1e-14
            for m in range(M):
                for s, k in enumerate(space.sm_counts):
                    want = nbytes[p, m] / (400e9 * min(1.0, k / 16.0) * (0.6 + 0.4 * f / 2000.0))
                    assert abs(t["tc"][p, fi, m, s] / want - 1) < 1e-14
                    assert abs(t["pc"][p, fi, m, s] / (cpow[p, m] * k / 32.0) - 1) < 1e-14
    assert t["t"].shape == (P, 3, N, 4) and t["tc"].shape == (P, 3, M, 3)
