"""CPU oracle for the short causal convolution (float64, plain numpy).

TEST INFRASTRUCTURE ONLY, like the rest of this package: nothing on the product path imports it.
"""
from __future__ import annotations

import numpy as np

from .gnorm import act


def _whole(x, state, length):
    """The inputs of a sequence [H, length] behind those of its state."""
    return np.concatenate([state, x[:, :length]], 1)


def short_fwd(x, k, bias, name, state=None, lengths=None):
    """y [B, H, N], last [B, H, taps - 1]."""
    B, H, N = x.shape
    W = k.shape[1]
    y, last = np.zeros((B, H, N)), np.zeros((B, H, W - 1))
    for b in range(B):
        n = N if lengths is None else int(np.clip(lengths[b], 0, N))
        w = _whole(x[b], np.zeros((H, W - 1)) if state is None else state[b], n)
        for t in range(n):
            z = bias + sum(k[:, j] * w[:, W - 1 + t - j] for j in range(W))
            y[b, :, t] = act(z, name)[0]
        last[b] = w[:, n:]
    return y, last


def short_bwd(dy, x, k, bias, name, state=None, lengths=None, dlast=None):
    """dx, dk, dbias, dstate."""
    B, H, N = x.shape
    W = k.shape[1]
    dx, dk, dbias, dstate = np.zeros((B, H, N)), np.zeros((H, W)), np.zeros(H), np.zeros((B, H, W - 1))
    for b in range(B):
        n = N if lengths is None else int(np.clip(lengths[b], 0, N))
        w = _whole(x[b], np.zeros((H, W - 1)) if state is None else state[b], n)
        dw = np.zeros_like(w)
        if dlast is not None:
            dw[:, n:] += dlast[b]
        for t in range(n):
            z = bias + sum(k[:, j] * w[:, W - 1 + t - j] for j in range(W))
            dz = dy[b, :, t] * act(z, name)[1]
            dbias += dz
            for j in range(W):
                dw[:, W - 1 + t - j] += k[:, j] * dz
                dk[:, j] += dz * w[:, W - 1 + t - j]
        dstate[b], dx[b, :, :n] = dw[:, :W - 1], dw[:, W - 1:]
    return dx, dk, dbias, dstate
