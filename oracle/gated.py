"""Gated feed-forward projections and their gradient (oracle), in float64."""
from __future__ import annotations

import numpy as np


def sigma(act: str, x):
    """The activation is x * sigma(x)."""
    x = np.asarray(x, np.float64)
    u = x if act == "silu" else 2.0 * np.sqrt(2.0 / np.pi) * (x + 0.044715 * x ** 3)
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-u))


def argument(act: str, x):
    """sigma's argument and its derivative."""
    x = np.asarray(x, np.float64)
    if act == "silu":
        return x, np.ones_like(x)
    c = 2.0 * np.sqrt(2.0 / np.pi)
    return c * (x + 0.044715 * x ** 3), c * (1.0 + 3.0 * 0.044715 * x ** 2)


def activation(act: str, x):
    """act(x) and act'(x)."""
    s = sigma(act, x)
    return x * s, s + x * s * (1.0 - s) * argument(act, x)[1]


def forward(x, w, b, act: str):
    """H and the pre-activations [G | U]; w [2 N, K]: gate rows, then the others."""
    pre = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if b is not None:
        pre = pre + b
    g, u = np.split(pre, 2, axis=1)
    return activation(act, g)[0] * u, pre


def backward(dh, pre, act: str):
    """The cotangent of the pre-activations from that of H."""
    g, u = np.split(np.asarray(pre, np.float64), 2, axis=1)
    a, d = activation(act, g)
    return np.concatenate([dh * u * d, dh * a], axis=1)
