"""Rows of e2m1 codes with block scales, in plain fp64 numpy: the definitions in
include/dart_cache.h."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# e4m3 without its sign and its NaN: code i stands for E4M3[i]
E4M3 = np.array([i * 2.0 ** -9 for i in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1])


def nearest(grid, x):
    """Index of the grid's value next to x >= 0, the even one of two as near."""
    hi = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    a, b = x - grid[hi - 1], grid[hi] - x
    return np.where((a < b) | ((a == b) & (hi % 2 == 1)), hi - 1, hi)


def quantise(x):
    """codes [..., 128] (0 .. 15), block codes [..., 8] (e4m3) and scales [...]
    of rows x [..., 128]."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    top = np.where(fine, np.abs(x), 0.0).max(-1)
    scale = np.where(top > 0, 2.0 ** np.maximum(np.frexp(top)[1] - 11, -120), 1.0)
    y = np.where(fine, x, 0.0).reshape(*x.shape[:-1], 8, 16) / scale[..., None, None]
    block = nearest(E4M3, np.abs(y).max(-1) / 6.0)
    value = E4M3[block][..., None]
    z = np.divide(np.abs(y), value, out=np.zeros_like(y), where=value > 0)
    code = nearest(E2M1, np.minimum(z, 6.0)) + 8 * np.signbit(x).reshape(y.shape)
    block = np.where(fine.reshape(y.shape).all(-1), block, 0x7F)
    return code.reshape(x.shape).astype(np.uint8), block.astype(np.uint8), scale


def values(code, block, scale):
    """What codes, block codes and scales stand for."""
    b = np.append(E4M3, np.nan)[block]
    v = np.where(code < 8, E2M1[code & 7], -E2M1[code & 7]).reshape(*code.shape[:-1], 8, 16)
    return (v * b[..., None] * np.asarray(scale, np.float64)[..., None, None]).reshape(code.shape)


def pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def unpack(byte):
    return np.stack([byte & 15, byte >> 4], -1).reshape(*byte.shape[:-1], 2 * byte.shape[-1])
