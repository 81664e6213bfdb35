"""CPU oracle for dropout masks that are drawn by a counter-based generator and never stored (plain numpy integers and float64).

TEST INFRASTRUCTURE ONLY, like the rest of this package: nothing on the product path imports it.

Philox4x32 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): each round maps the counter
(c0, c1, c2, c3) to (hi(M1 c2) ^ c1 ^ k0, lo(M1 c2), hi(M0 c0) ^ c3 ^ k1, lo(M0 c0)), and the key grows by (W0, W1) between rounds.
Entry i of a tensor has half i mod 8 (low half of a word first) of the four words of the counter (i div 8, call) under the key `seed`,
and is kept iff these 16 bits are at least T = floor(65536 p + 1/2).
"""
from __future__ import annotations

import numpy as np

M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85


def philox(counter, key, rounds: int = 7):
    """counter: four arrays (or numbers) of 32-bit words, key: two numbers."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k0, k1 = (int(x) for x in key)
    low, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(M0), c[2] * np.uint64(M1)
        c = [(b >> shift) ^ c[1] ^ np.uint64(k0), b & low, (a >> shift) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + W0) % 2 ** 32, (k1 + W1) % 2 ** 32
    return c


def threshold(p: float) -> int:
    return int(np.floor(float(np.float32(p)) * 65536 + 0.5))


def bits(entries, seed: int, call: int):
    """The 16 bits of the entries with these numbers."""
    i = np.asarray(entries, dtype=np.uint64)
    block, at = i // np.uint64(8), i % np.uint64(8)
    counter = (block % np.uint64(2 ** 32), block // np.uint64(2 ** 32), call % 2 ** 32, call // 2 ** 32)
    words = [np.broadcast_to(w, i.shape) for w in philox(counter, (seed % 2 ** 32, seed // 2 ** 32))]
    word = np.choose((at // np.uint64(2)).astype(np.int64), words)
    return np.where(at % np.uint64(2) == 0, word % np.uint64(65536), word // np.uint64(65536)).astype(np.int64)


def factors(entries, p: float, seed: int, call: int):
    """m of these entries."""
    T = threshold(p)
    scale = 0.0 if T >= 65536 else 65536.0 / (65536 - T)
    return np.where(bits(entries, seed, call) >= T, scale, 0.0)


def mask(shape, p: float, seed: int, call: int, tie: int = 1):
    """m over a tensor, runs of `tie` entries sharing a value."""
    n = int(np.prod(shape))
    return factors(np.arange(n) // tie, p, seed, call).reshape(shape)


def dropout(x, m, residual=None):
    """residual + m x; a dropped x counts for nothing, whatever it holds."""
    y = np.where(m == 0, 0.0, np.where(m == 0, 0.0, x) * m)
    return y if residual is None else y + residual
