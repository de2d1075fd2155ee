"""Dropout from a counter-based generator (oracle): Philox4x32-10 (Salmon, Moraes, Dror and
Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011) in Python integers' terms."""
from __future__ import annotations

import numpy as np

LOW = np.uint64(0xFFFFFFFF)


def philox(counter, key):
    """Ten rounds over counters of four words (arrays of uint64 below 2^32), key of two."""
    c = [np.asarray(v, np.uint64) for v in counter]
    k = [int(v) for v in key]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & LOW,
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & LOW]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def kept(n: int, p: float, seed: int, step: int, site: int, first: int = 0):
    """Which of the values first .. first + n - 1 stay (first a multiple of 8), and the
    factor of those."""
    block = np.arange(first // 8, (first + n + 7) // 8, dtype=np.uint64)
    fill = lambda v: np.full(len(block), v, np.uint64)
    w = philox([block, fill(site), fill(step % 2 ** 32), fill(step >> 32)], [seed % 2 ** 32, seed >> 32])
    draws = np.stack([v for word in w for v in (word & np.uint64(0xFFFF), word >> np.uint64(16))], axis=1)
    least = int(np.rint(p * 65536))
    return draws.reshape(-1)[:n] >= least, 65536.0 / (65536 - least)
