"""CPU oracle for the embedding and its gradient (float64, plain numpy).

TEST INFRASTRUCTURE ONLY, like the rest of this package: nothing on the product path imports it.
"""
from __future__ import annotations

import numpy as np


def embed_fwd(ids, E, scale: float, first: bool, m=None):
    """y [B, N, H] ([B, H, N] if `first`) = m . scale . E[ids]; ids outside the table give zeros."""
    B, N = ids.shape
    V, H = E.shape
    y = np.zeros((B, N, H))
    for b in range(B):
        for t in range(N):
            if 0 <= ids[b, t] < V:
                y[b, t] = scale * E[ids[b, t]]
    y = y.transpose(0, 2, 1) if first else y
    return y if m is None else np.where(m == 0, 0.0, y * m)


def embed_bwd(dy, ids, V: int, scale: float, first: bool, m=None):
    """dE [V, H]: what reaches each row of the table."""
    g = dy if m is None else np.where(m == 0, 0.0, np.where(m == 0, 0.0, dy) * m)
    g = g.transpose(0, 2, 1) if first else g
    dE = np.zeros((V, g.shape[2]))
    for b in range(ids.shape[0]):
        for t in range(ids.shape[1]):
            if 0 <= ids[b, t] < V:
                dE[ids[b, t]] += g[b, t]
    return scale * dE
