"""Cross entropy of a linear layer's outputs and its gradient (oracle), in float64."""
from __future__ import annotations

import numpy as np


def forward(z, targets):
    """stats [M, 2] (the largest logit, ln of the sum of e^(z - it)) and the losses [M]
    of logits z.  A row of nothing but -inf: (-inf, 0) and loss inf; no target: 0."""
    z = np.asarray(z, np.float64)
    rows, V = z.shape
    t = np.asarray(targets)
    with np.errstate(all="ignore"):
        m = z.max(axis=1)
        empty = m == -np.inf
        s = np.exp(z - np.where(empty, 0.0, m)[:, None]).sum(axis=1)
        ln = np.where(empty, 0.0, np.log(np.where(empty, 1.0, s)))
        zt = z[np.arange(rows), np.clip(t, 0, V - 1)]
        loss = np.where(zt == -np.inf, np.inf, (m - zt) + ln)
        loss = np.where(np.isnan(ln), np.nan, loss)
    loss = np.where(t >= V, np.nan, np.where(t < 0, 0.0, loss))
    return np.stack([m, ln], axis=1), loss


def dlogits(z, targets, stats, g, scale: float):
    """scale g (p - [target]) per row; masked logits and rows without a target get 0, rows of
    NaN stats or a target outside the vocabulary NaN."""
    z = np.asarray(z, np.float64)
    rows, V = z.shape
    t = np.asarray(targets)
    with np.errstate(all="ignore"):
        empty = stats[:, 0] == -np.inf
        m, ln = (np.where(empty, 0.0, stats[:, i])[:, None] for i in range(2))
        p = np.exp((z - m) - ln)
    hot = np.arange(V) == t[:, None]
    f = np.where(t < 0, 0.0, np.where(t >= V, np.nan, scale * np.asarray(g, np.float64)))
    bad = (np.isnan(ln[:, 0]) | np.isnan(f))[:, None]
    return np.where((z == -np.inf) & ~bad, 0.0, np.where(bad, np.nan, (p - hot) * f[:, None]))


def mean_weights(targets):
    """The cotangents that the mean over the rows with a target has."""
    has = np.asarray(targets) >= 0
    return np.full(len(has), 1.0 / max(1, has.sum()))
