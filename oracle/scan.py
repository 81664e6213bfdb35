"""CPU oracle for the selective state space scan (float64, plain numpy): place by place, and backwards by the chain rule.

TEST INFRASTRUCTURE ONLY, like the rest of this package: nothing on the product path imports it.
"""
from __future__ import annotations

import numpy as np


def silu(z):
    q = 1.0 / (1.0 + np.exp(-z))
    return z * q, q * (1.0 + z * (1.0 - q))


def time_steps(delta, bias, softplus):
    """dt and its slope in delta, [B, H, N]."""
    w = delta if bias is None else delta + bias[:, None]
    if not softplus:
        return w, np.ones_like(w)
    return np.logaddexp(w, 0.0), 1.0 / (1.0 + np.exp(-w))


def inside(lengths, B, N):
    """[B, 1, N]: whether a place belongs to its sequence."""
    n = np.full(B, N) if lengths is None else np.clip(lengths, 0, N)
    return (np.arange(N) < n[:, None])[:, None]


def scan_fwd(u, delta, A, Bm, Cm, D=None, z=None, bias=None, softplus=True, state=None, lengths=None):
    """y [B, H, N], last [B, H, S], and the states in front of every place and behind the last, [N + 1, B, H, S]."""
    B, H, N = u.shape
    G, S = Bm.shape[1:3]
    there = inside(lengths, B, N)
    dt = np.where(there, time_steps(delta, bias, softplus)[0], 0.0)
    u = np.where(there, u, 0.0)
    Bm, Cm = (np.repeat(np.where(there[:, None], m, 0.0), H // G, 1) for m in (Bm, Cm))
    h = np.zeros((N + 1, B, H, S))
    if state is not None:
        h[0] = state
    y = np.zeros((B, H, N))
    for t in range(N):
        h[t + 1] = np.exp(dt[:, :, t, None] * A) * h[t] + (dt[:, :, t] * u[:, :, t])[..., None] * Bm[..., t]
        y[:, :, t] = (Cm[..., t] * h[t + 1]).sum(2)
    if D is not None:
        y = y + D[:, None] * u
    if z is not None:
        y = y * silu(np.where(there, z, 0.0))[0]
    return np.where(there, y, 0.0), h[N], h


def scan_bwd(dy, u, delta, A, Bm, Cm, D=None, z=None, bias=None, softplus=True, state=None, lengths=None, dlast=None):
    """A dict of du, ddelta, dA, dB, dC, dD, dz, dbias, dstate."""
    B, H, N = u.shape
    G, S = Bm.shape[1:3]
    there = inside(lengths, B, N)
    h = scan_fwd(u, delta, A, Bm, Cm, D, z, bias, softplus, state, lengths)[2]
    dt, rate = time_steps(delta, bias, softplus)
    dt, u, dy = np.where(there, dt, 0.0), np.where(there, u, 0.0), np.where(there, dy, 0.0)
    Bm, Cm = (np.repeat(np.where(there[:, None], m, 0.0), H // G, 1) for m in (Bm, Cm))
    D = np.zeros(H) if D is None else D
    dz = np.zeros_like(u)
    if z is not None:
        gate, slope = silu(np.where(there, z, 0.0))
        plain = np.einsum("bhsn,nbhs->bhn", Cm, h[1:]) + D[:, None] * u
        dz, dy = dy * plain * slope, dy * gate
    g = np.zeros((B, H, S)) if dlast is None else dlast.copy()
    out = {k: np.zeros_like(u) for k in ("du", "ddelta")}
    dA, dB, dC = np.zeros((H, S)), np.zeros((B, H, S, N)), np.zeros((B, H, S, N))
    for t in reversed(range(N)):
        g = g + dy[:, :, t, None] * Cm[..., t]
        a = np.exp(dt[:, :, t, None] * A)
        dC[..., t] = dy[:, :, t, None] * h[t + 1]
        dB[..., t] = g * (dt[:, :, t] * u[:, :, t])[..., None]
        kept = g * a * h[t]
        dA += (kept * dt[:, :, t, None]).sum(0)
        gB = (g * Bm[..., t]).sum(2)
        out["du"][:, :, t] = dt[:, :, t] * gB + D * dy[:, :, t]
        out["ddelta"][:, :, t] = ((kept * A).sum(2) + u[:, :, t] * gB) * np.where(there, rate, 0.0)[:, :, t]
        g = g * a
    fold = lambda m: m.reshape(B, G, H // G, S, N).sum(2)  # noqa: E731
    out.update(dA=dA, dB=fold(dB), dC=fold(dC), dD=(dy * u).sum((0, 2)), dz=dz, dbias=out["ddelta"].sum((0, 2)), dstate=g)
    return out
