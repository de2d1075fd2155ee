"""Rotary positions with several axes (oracle), in float64 from the definition.

A head's values hold one section of 2 n_a values per axis; pair i of axis a
turns by pos[a] * base_a^(-i / n_a) radians; what lies behind the sections is
not turned."""
from __future__ import annotations

import numpy as np


def pair_columns(pairs, interleaved: bool):
    """[(axis, i, first column, second column)] of every pair of a head."""
    out, o = [], 0
    for a, n in enumerate(pairs):
        for i in range(n):
            out.append((a, i, o + 2 * i, o + 2 * i + 1) if interleaved else (a, i, o + i, o + n + i))
        o += 2 * n
    return out


def turn(x, pos, pairs, base, interleaved: bool, heads_rot: int, hd: int, back: bool = False):
    """x [rows, heads * hd]; pos [pos_rows, axes], row r at pos[r % pos_rows].
    The first heads_rot heads are turned, the others returned as they are."""
    x = np.asarray(x, np.float64)
    rows = x.shape[0]
    y = x.reshape(rows, -1, hd).copy()
    h = x.reshape(rows, -1, hd)
    p = np.asarray(pos, np.float64)[np.arange(rows) % len(pos)]
    for a, i, c0, c1 in pair_columns(pairs, interleaved):
        ang = p[:, a] * float(base[a]) ** (-i / pairs[a])
        c, s = np.cos(ang)[:, None], np.sin(ang)[:, None] * (-1.0 if back else 1.0)
        x0, x1 = h[:, :heads_rot, c0], h[:, :heads_rot, c1]
        y[:, :heads_rot, c0] = x0 * c - x1 * s
        y[:, :heads_rot, c1] = x1 * c + x0 * s
    return y.reshape(rows, -1)
