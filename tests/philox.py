"""Philox4x32 with 10 rounds in numpy, written from its definition, and the numbers that dropout takes from it."""

import numpy as np


def philox4x32(counter, key, rounds=10):
    """counter: four arrays or numbers, key: two numbers; four arrays of uint32."""
    x = [np.asarray(v, dtype=np.uint64) for v in counter]
    k0, k1 = (int(v) for v in key)
    low = np.uint64(0xFFFFFFFF)
    for _ in range(rounds):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ x[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return [v.astype(np.uint32) for v in x]


def dropout_numbers(seed, step, site, rows, cols, row0=0):
    """(rows, cols) of 16 random bits: those of rows row0 .. of a dropout."""
    groups = (cols + 7) // 8
    shape = rows, groups
    seed &= (1 << 64) - 1
    words = philox4x32([np.broadcast_to(np.arange(groups), shape), np.broadcast_to(np.arange(row0, row0 + rows)[:, None], shape),
                        np.full(shape, site), np.full(shape, step & 0xFFFFFFFF)], [seed & 0xFFFFFFFF, seed >> 32])
    halves = [h for w in words for h in (w & 0xFFFF, w >> 16)]
    return np.stack(halves, -1).reshape(rows, groups * 8)[:, :cols]
