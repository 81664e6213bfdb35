"""CPU oracle for group norm with an activation, channels last (float64, plain numpy).

TEST INFRASTRUCTURE ONLY, like the rest of this package: nothing on the product path imports it.
"""
from __future__ import annotations

import math

import numpy as np


def act(z, name: str):
    """act(z) and its slope (relu: slope 0 at 0)."""
    if name == "silu":
        q = 1.0 / (1.0 + np.exp(-z))
        return z * q, q * (1.0 + z * (1.0 - q))
    if name == "gelu":
        q = 0.5 * np.vectorize(math.erfc, otypes=[float])(-z / math.sqrt(2.0))
        return z * q, q + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if name == "relu":
        return np.maximum(z, 0.0), (z > 0).astype(float)
    assert name == "none"
    return z, np.ones_like(z)


def statistics(x, G: int, eps: float):
    """mean, rstd [B, G] of x [B, S, C]."""
    B, S, C = x.shape
    g = x.reshape(B, S, G, C // G)
    mean = g.mean(axis=(1, 3))
    var = ((g - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    return mean, 1.0 / np.sqrt(var + eps)


def gnorm_fwd(x, gamma, beta, G: int, eps: float, name: str):
    """y, mean, rstd."""
    B, S, C = x.shape
    mean, rstd = statistics(x, G, eps)
    xhat = (x - np.repeat(mean, C // G, 1)[:, None]) * np.repeat(rstd, C // G, 1)[:, None]
    return act(xhat * gamma + beta, name)[0], mean, rstd


def gnorm_bwd(dy, x, gamma, beta, G: int, eps: float, name: str):
    """dx, dgamma, dbeta."""
    B, S, C = x.shape
    mean, rstd = (np.repeat(a, C // G, 1)[:, None] for a in statistics(x, G, eps))
    xhat = (x - mean) * rstd
    dz = dy * act(xhat * gamma + beta, name)[1]
    t = gamma * dz
    of = lambda a: np.repeat(a.reshape(B, S, G, C // G).mean(axis=(1, 3)), C // G, 1)[:, None]  # noqa: E731
    return rstd * (t - of(t) - xhat * of(t * xhat)), (dz * xhat).sum(axis=(0, 1)), dz.sum(axis=(0, 1))
