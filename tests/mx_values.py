"""Rows in 4 bits by their definition, in numpy: what the tests of them compare with."""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def blocks_of(k):
    return (k + 31) // 32


def quantized(x):
    """(q uint8 [rows, 16 blocks], scale uint8 [rows, blocks]) of a float tensor."""
    x = x.double().numpy()
    rows, k = x.shape
    b = blocks_of(k)
    x = np.concatenate([x, np.zeros((rows, b * 32 - k))], 1).reshape(rows, b, 32)
    bad = ~np.isfinite(x).all(2)
    x = np.where(bad[:, :, None], 0.0, x)
    most = np.abs(x).max(2)
    code = np.where(most > 0, np.maximum(np.frexp(most)[1] - 1 - 2, -127) + 127, 0)
    y = np.abs(x) / np.ldexp(1.0, code - 127)[:, :, None]
    # the nearest of the grid, ties to the even place, past the last to it
    dist = np.abs(y[..., None] - GRID)
    place = np.argmin(np.where(dist == dist.min(-1, keepdims=True), np.arange(8) % 2, 2), -1)
    # (of the nearest, one or two neighbours: the first even place, else the odd one)
    nibble = (place | (np.signbit(x).astype(np.int64) << 3)).reshape(rows, -1, 2)
    nibble = np.where(np.repeat(bad, 16, axis=1)[:, :, None], 0, nibble)
    q = (nibble[:, :, 0] | nibble[:, :, 1] << 4).astype(np.uint8)
    return q, np.where(bad, 255, code).astype(np.uint8)


def values(q, scale):
    """What they stand for, float64 [rows, 32 blocks]."""
    n = np.stack([q & 15, q >> 4], 2).reshape(q.shape[0], -1)
    v = np.where(n & 8, -1.0, 1.0) * GRID[n & 7]
    s = np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    return v * np.repeat(s, 32, axis=1)


def draw(rows, k, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, k, generator=g) * torch.exp(2 * torch.randn(rows, 1, generator=g))
    return x.to(dtype)
