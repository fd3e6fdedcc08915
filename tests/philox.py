"""Philox4x32 with ten rounds in numpy, from its definition (Salmon, Moraes, Dror
and Shaw, 2011)."""
import numpy as np


def block(counter, key):
    """Four words for each counter: counter [4 arrays of uint32], key (k0, k1)."""
    x = [np.asarray(c, dtype=np.uint64) for c in counter]
    k = [int(k) for k in key]
    low, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [b >> shift ^ x[1] ^ np.uint64(k[0]), b & low, a >> shift ^ x[3] ^ np.uint64(k[1]),
             a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return x


def words(seed, offset, count):
    """Words 0..count-1: four a counter, from `offset` (64 bits) on."""
    with np.errstate(over="ignore"):
        c = np.uint64(offset) + np.arange((count + 3) // 4, dtype=np.uint64)
    zero = np.zeros_like(c)
    x = block([c & np.uint64(0xFFFFFFFF), c >> np.uint64(32), zero, zero],
              (seed & 0xFFFFFFFF, seed >> 32))
    return np.stack(x, 1).reshape(-1)[:count]
