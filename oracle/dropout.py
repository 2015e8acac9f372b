"""Dropout from a counter-based generator (numpy, Python's whole numbers).

TEST INFRASTRUCTURE ONLY -- see oracle/__init__.py.

Philox 4x32 with ten rounds, as in Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as
easy as 1, 2, 3" (SC 2011): one round takes (c0, c1, c2, c3) with the key (k0, k1) to
(hi(M1 c2) ^ c1 ^ k0, lo(M1 c2), hi(M0 c0) ^ c3 ^ k1, lo(M0 c0)); the key then grows by the
increments.
"""

import numpy as np

__all__ = ["philox", "words", "dropout_keep", "dropout_fwd"]

_MASK = (1 << 32) - 1


def philox(counter, key):
    """The four words of one block: counter and key are lists of 32-bit whole numbers."""
    c, k = [int(v) for v in counter], [int(v) for v in key]
    for _ in range(10):
        p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [q >> 32 ^ c[1] ^ k[0], q & _MASK, p >> 32 ^ c[3] ^ k[1], p & _MASK]
        k = [(k[0] + 0x9E3779B9) & _MASK, (k[1] + 0xBB67AE85) & _MASK]
    return c


def words(first, n, seed, offset):
    """Words first .. first + n of the stream of (seed, offset)."""
    seed, offset = int(seed) % 2 ** 64, int(offset) % 2 ** 64
    out = []
    for b in range(first // 4, (first + n + 3) // 4):
        out += philox([b & _MASK, b >> 32, offset & _MASK, offset >> 32], [seed & _MASK, seed >> 32])
    at = first - 4 * (first // 4)
    return np.array(out[at:at + n], dtype=np.uint64)


def dropout_keep(n, p, seed, offset, first=0):
    return words(first, n, seed, offset) >= round(p * 2 ** 32)


def dropout_fwd(x, p, seed, offset=0, residual=None):
    x = np.asarray(x, dtype=np.float64)
    y = np.where(dropout_keep(x.size, p, seed, offset).reshape(x.shape), x / (1.0 - p), 0.0)
    return y if residual is None else residual + y
