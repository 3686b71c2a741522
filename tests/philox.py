"""Dropout's masks by the definition: Philox4x32-10 in whole numbers, number by number."""

import numpy as np
import torch


def philox(counter, key):
    """Four words of a counter of four and a key of two (numbers or arrays of them)."""
    c, k = [np.asarray(x, dtype=np.uint64) for x in counter], list(key)
    low = np.uint64(0xFFFFFFFF)
    half = np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]),
             a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def bits(rows, width, seed, offset, row0=0):
    """The 16 bits of each value, [rows][width]."""
    groups = -(-width // 8)
    g = np.broadcast_to(np.arange(groups), (rows, groups))
    r = np.broadcast_to(np.arange(row0, row0 + rows)[:, None], (rows, groups))
    o = [np.full((rows, groups), x) for x in (offset % 2 ** 32, offset >> 32)]
    words = np.stack(philox([g, r, *o], [seed % 2 ** 32, seed >> 32]), -1)
    halves = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], -1)
    return halves.reshape(rows, groups * 8)[:, :width].astype(np.int64)


def factor(rows, width, p, seed, offset, row0=0):
    """What each value is multiplied by, in 64 bits: 0, or the kept ones' factor."""
    cut = int(round(p * 65536))
    kept = torch.from_numpy(bits(rows, width, seed, offset, row0) >= cut)
    return torch.where(kept, 65536.0 / max(65536 - cut, 1), 0.0).double()
