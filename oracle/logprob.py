"""Log probabilities of given tokens, entropy and top alternatives, and their
gradient at the logits (oracle), in float64 from the definitions."""
from __future__ import annotations

import numpy as np


def forward(z, targets, k: int):
    """stats [rows, 2] (the largest logit and ln of the sum of e^(z - it)), logp,
    entropy [rows], top_logp and top_idx [rows, k]."""
    z = np.asarray(z, np.float64)
    rows, V = z.shape
    t = np.asarray(targets)
    with np.errstate(all="ignore"):
        m = z.max(axis=1)
        bad = ~(m < np.inf)                       # NaN or +inf in the row
        empty = m == -np.inf
        d = z - np.where(empty | bad, 0.0, m)[:, None]
        e = np.where(bad[:, None], 1.0, np.exp(np.where(bad[:, None], 0.0, d)))
        S = np.where(empty, 1.0, e.sum(axis=1))
        lp = np.where(empty[:, None], -np.inf, d - np.log(S)[:, None])
        p = e / S[:, None]
        ent = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum(axis=1)
        ent = np.where(bad, np.nan, np.where(empty, 0.0, ent))
        stats = np.where(bad[:, None], np.nan, np.stack([m, np.log(S)], axis=1))
        lp[bad] = np.nan
        own = lp[np.arange(rows), np.clip(t, 0, V - 1)]
        logp = np.where(t < 0, 0.0, np.where(t >= V, np.nan, own))
    # NaN above all, equal values by the lower column
    rank = np.where(np.isnan(z), np.inf, z)
    order = np.lexsort((np.broadcast_to(np.arange(V), z.shape), -rank, ~np.isnan(z)), axis=1)[:, :k]
    return stats, logp, ent, np.take_along_axis(lp, order, axis=1), order


def backward(z, targets, stats, entropy, top_idx, g_logp, g_entropy, g_top, scale):
    """dZ before its rounding; stats and entropy as given (any cotangent may be
    None).  Also returns the sum of the magnitudes that each element adds up."""
    z = np.asarray(z, np.float64)
    rows, V = z.shape
    stats = np.asarray(stats, np.float64)
    empty = stats[:, 0] == -np.inf
    with np.errstate(all="ignore"):
        lp = (z - np.where(empty, 0.0, stats[:, 0])[:, None]) - stats[:, 1:]
        p = np.exp(lp)
    up, mag = np.zeros(rows), np.zeros(rows)
    own = np.zeros((rows, V))
    at = np.arange(rows)
    if g_logp is not None:
        t = np.asarray(targets)
        g = np.where(t < 0, 0.0, np.asarray(g_logp, np.float64))
        np.add.at(own, (at, np.clip(t, 0, V - 1)), np.where(t < V, g, 0.0))
        up += np.where(t >= V, np.nan, g)
        mag += np.abs(g)
    if g_top is not None:
        for i in range(np.shape(top_idx)[1]):
            g = np.asarray(g_top, np.float64)[:, i]
            np.add.at(own, (at, top_idx[:, i]), g)
            up += g
            mag += np.abs(g)
    total = np.abs(own) + p * mag[:, None]
    with np.errstate(all="ignore"):
        d = own - p * up[:, None]
        if g_entropy is not None:
            ge, H = np.asarray(g_entropy, np.float64)[:, None], np.asarray(entropy, np.float64)[:, None]
            term = np.where(p > 0, p * (np.where(p > 0, lp, 0.0) + H), 0.0)
            d = d - ge * term
            total = total + np.abs(ge) * np.where(p > 0, p * (np.abs(np.where(p > 0, lp, 0.0)) + np.abs(H)), 0.0)
        d = np.where((z == -np.inf) | empty[:, None], 0.0, d)
        d = np.where((np.isnan(stats).any(axis=1) | np.isnan(up))[:, None], np.nan, d)
    return scale * d, abs(scale) * total
