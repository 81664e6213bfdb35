"""CPU oracle for the dense product between layers (float64, plain numpy).

TEST INFRASTRUCTURE ONLY, like the rest of this package: nothing on the product path imports it.
"""
from __future__ import annotations

import numpy as np

from .gnorm import act


def last(t, first: bool):
    """[B, C, N] or [B, N, C] -> [B, N, C]."""
    return t.transpose(0, 2, 1) if first else t


def linear_fwd(x, W, bias, name, x_first=False, y_first=False, residual=None):
    z = last(x, x_first) @ W.T + bias
    y = last(act(z, name)[0], y_first)
    return y if residual is None else y + residual


def linear_bwd(dy, x, W, bias, name, x_first=False, y_first=False):
    """dx, dW, dbias, dz [B, N, M]."""
    rows = last(x, x_first)
    dz = last(dy, y_first) * act(rows @ W.T + bias, name)[1]
    return last(dz @ W, x_first), np.einsum("bnm,bnk->mk", dz, rows), dz.sum((0, 1)), dz
