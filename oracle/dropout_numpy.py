"""Dropout from a counter-based generator, from its definition, in numpy.

Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011) word by word;
the block of eight neighbouring elements of a row is the counter (col // 8, row, sequence low, sequence high), the
key is the seed.  Written apart from the CUDA code and used by the tests only.
"""
from __future__ import annotations

import numpy as np

M0, M1 = np.uint64(0xD2511F53), np.uint64(0xCD9E8D57)
W0, W1 = 0x9E3779B9, 0xBB67AE85
LOW, SHIFT = np.uint64(0xFFFFFFFF), np.uint64(32)


def philox4x32_10(counter, key):
    """counter: four arrays (or numbers) of 32-bit words; key: two numbers.  Returns four uint64 arrays of 32-bit words."""
    x = [np.asarray(c, dtype=np.uint64) for c in counter]
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(10):
        p, q = x[0] * M0, x[2] * M1
        x = [(q >> SHIFT) ^ x[1] ^ np.uint64(k0), q & LOW, (p >> SHIFT) ^ x[3] ^ np.uint64(k1), p & LOW]
        k0, k1 = (k0 + W0) & 0xFFFFFFFF, (k1 + W1) & 0xFFFFFFFF
    return x


def threshold(p: float) -> int:
    """Drop rate in 1/65536, halves up."""
    return int(np.floor(p * 65536.0 + 0.5))


def lanes(rows: int, cols: int, seed: int, sequence: int, first_row: int = 0, first_block: int = 0) -> np.ndarray:
    """16-bit random lane of every element, [rows, cols]; the first row and the first block of eight may be given."""
    blocks = (cols + 7) // 8
    row = np.repeat(np.arange(first_row, first_row + rows, dtype=np.uint64)[:, None], blocks, axis=1)
    block = np.repeat(np.arange(first_block, first_block + blocks, dtype=np.uint64)[None, :], rows, axis=0)
    words = philox4x32_10([block, row, sequence & 0xFFFFFFFF, (sequence >> 32) & 0xFFFFFFFF],
                          [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF])
    out = np.empty((rows, blocks, 8), dtype=np.uint32)
    for j in range(4):
        out[:, :, 2 * j] = words[j] & np.uint64(0xFFFF)
        out[:, :, 2 * j + 1] = words[j] >> np.uint64(16)
    return out.reshape(rows, 8 * blocks)[:, :cols]


def keep_mask(rows: int, cols: int, p: float, seed: int, sequence: int, first_row: int = 0, first_block: int = 0) -> np.ndarray:
    return lanes(rows, cols, seed, sequence, first_row, first_block) >= threshold(p)


def scale(p: float) -> float:
    t = threshold(p)
    return 65536.0 / (65536 - t) if t < 65536 else 0.0


def dropout(x, p, seed, sequence, residual=None):
    """float64 [rows, cols] in, float64 out."""
    x = np.asarray(x, dtype=np.float64)
    y = np.zeros_like(x)
    keep = keep_mask(x.shape[0], x.shape[1], p, seed, sequence)
    y[keep] = x[keep] * scale(p)
    return y if residual is None else np.asarray(residual, dtype=np.float64) + y
