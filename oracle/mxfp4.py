"""Microscaled 4-bit values (blocks of 32, e2m1 elements, one power of two per block), restated in numpy from the format's
definition: search over the grid instead of bit arithmetic, and the scale images read back element by element."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def quantize(x: np.ndarray):
    """(codes int [rows, blocks, 32], exponents int [rows, blocks], 128 for a block that is NaN) of x [rows, C]."""
    rows, c = x.shape
    blocks = -(-c // BLOCK)
    v = np.zeros((rows, blocks * BLOCK))
    v[:, :c] = x
    v = v.reshape(rows, blocks, BLOCK)
    bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    top = np.abs(v).max(-1)
    e = np.full(top.shape, -127, dtype=np.int64)
    for k in range(-126, 126):                       # the largest k with 2^(k+2) <= top
        e[top >= 2.0 ** (k + 2)] = k
    a = np.abs(v) / (2.0 ** e.astype(np.float64))[..., None]
    far = np.abs(a[..., None] - GRID)
    near = far.min(-1, keepdims=True)
    even_first = np.array([0, 2, 4, 6, 1, 3, 5, 7])  # of two equally near codes the even one
    codes = even_first[np.argmax((far == near)[..., even_first], axis=-1)]
    codes = np.where(np.signbit(v), codes + 8, codes)
    return codes, np.where(bad, 128, e)


def values(codes: np.ndarray, e: np.ndarray, c: int) -> np.ndarray:
    """The numbers that codes and exponents stand for, float64 [rows, c]."""
    q = np.where(codes >= 8, -1.0, 1.0) * GRID[codes & 7]
    scale = np.where(e == 128, np.nan, 2.0 ** e.astype(np.float64))
    return (q * scale[..., None]).reshape(codes.shape[0], -1)[:, :c]


def code_bytes(codes: np.ndarray) -> np.ndarray:
    """[rows, blocks * 16] bytes: two channels per byte, the lower one in the low half."""
    flat = codes.reshape(codes.shape[0], -1)
    return (flat[:, 0::2] | (flat[:, 1::2] << 4)).astype(np.uint8)


def scale_image_index(row: int, block: int, blocks: int) -> int:
    """Where the scale of a row's block stands in the scales' bytes."""
    chunks = -(-blocks // 4)
    image = (row // 128) * chunks + block // 4
    return image * 512 + (row % 32) * 16 + (row % 128 // 32) * 4 + block % 4
