"""Norms of queries and keys for each head with rotary positions (oracle), in float64."""
from __future__ import annotations

import numpy as np

from oracle.rotary import turn


def _gains(wq, wk, heads_q: int, heads_k: int, hd: int):
    one = np.ones(hd)
    return np.stack([one if wq is None else np.asarray(wq, np.float64)] * heads_q
                    + [one if wk is None else np.asarray(wk, np.float64)] * heads_k)


def _root(h, eps):
    with np.errstate(divide="ignore"):
        return 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)


def forward(x, wq, wk, eps, pos, pairs, base, interleaved, heads_q, heads_k, hd):
    x = np.asarray(x, np.float64)
    rows, rot = len(x), heads_q + heads_k
    h = x.reshape(rows, -1, hd)[:, :rot]
    n = x.reshape(rows, -1, hd).copy()
    n[:, :rot] = h * _root(h, eps) * _gains(wq, wk, heads_q, heads_k, hd)
    return turn(n.reshape(rows, -1), pos, pairs, base, interleaved, rot, hd), n.reshape(rows, -1)


def backward(x, dy, wq, wk, eps, pos, pairs, base, interleaved, heads_q, heads_k, hd):
    """dx, dwq, dwk, and the unturned cotangents."""
    rows, rot = len(x), heads_q + heads_k
    h = np.asarray(x, np.float64).reshape(rows, -1, hd)[:, :rot]
    dn = turn(dy, pos, pairs, base, interleaved, rot, hd, True)
    d = dn.reshape(rows, -1, hd)[:, :rot]
    r, w = _root(h, eps), _gains(wq, wk, heads_q, heads_k, hd)
    dx = dn.reshape(rows, -1, hd).copy()
    dx[:, :rot] = r * (w * d - h * r * r * (w * d * h).mean(-1, keepdims=True))
    dw = d * h * r
    return dx.reshape(rows, -1), dw[:, :heads_q].sum((0, 1)), dw[:, heads_q:].sum((0, 1)), dn
