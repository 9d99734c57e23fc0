"""Plain reference of MXFP4 matrices -- TEST INFRASTRUCTURE.

Only ``tests/`` may import this module; the product never does, and this module
imports nothing from it.

Rows of E2M1 elements (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) in blocks of
32, each with the scale 2^(b - 127), b = max(E - 2, 0) for the biased exponent E of
the block's largest magnitude as a float.  Rows are padded with zeros to a multiple
of 128 columns.  Every step is written out plainly in float64: the grid is
enumerated and an element goes to the nearest value, ties to the even code.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def padded(cols: int) -> int:
    return -(-cols // 128) * 128


def encode(v):
    """Codes [rows][P] (one per element, 0..15) and scale bytes [rows][P / 32] of a 2-D
    array, read as fp32."""
    v = np.asarray(v, np.float32)
    rows, cols = v.shape
    P = padded(cols)
    x = np.zeros((rows, P), np.float32)
    x[:, :cols] = v
    blocks = x.reshape(rows, P // 32, 32)
    bits = blocks.view(np.uint32) & np.uint32(0x7FFFFFFF)
    E = (bits.max(axis=2) >> 23).astype(np.int64)
    byte = np.where(E == 255, 255, np.maximum(E - 2, 0))
    bad = byte == 255
    with np.errstate(invalid="ignore", over="ignore"):
        a = np.abs(blocks.astype(np.float64)) * np.exp2(127.0 - np.where(bad, 127, byte))[..., None]
    a = np.where(bad[..., None], 0.0, a)
    dist = np.abs(a[..., None] - GRID)
    best = dist.min(axis=-1, keepdims=True)
    near = dist == best                                  # one value, or two at a tie
    lo = near.argmax(axis=-1)
    hi = 7 - near[..., ::-1].argmax(axis=-1)
    code = np.where(lo % 2 == 0, lo, hi)
    code = np.where(np.signbit(blocks) & ~bad[..., None], code + 8, code)
    return code.reshape(rows, P).astype(np.uint8), byte.astype(np.uint8)


def pack(code) -> np.ndarray:
    return (code[:, ::2] | (code[:, 1::2] << 4)).astype(np.uint8)


def unpack(packed) -> np.ndarray:
    out = np.empty((packed.shape[0], 2 * packed.shape[1]), np.uint8)
    out[:, ::2], out[:, 1::2] = packed & 15, packed >> 4
    return out


def values(code, byte, cols: int) -> np.ndarray:
    """The values of codes (one per element) and scale bytes, float64."""
    code, byte = np.asarray(code, np.int64), np.asarray(byte, np.int64)
    v = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7]
    s = np.where(byte == 255, np.nan, np.exp2(byte - 127.0))
    return (v.reshape(v.shape[0], -1, 32) * s[..., None]).reshape(v.shape[0], -1)[:, :cols]


def rounded(v) -> np.ndarray:
    """The values that a 2-D array has as an MXFP4 matrix, float64."""
    code, byte = encode(v)
    return values(code, byte, np.asarray(v).shape[1])
