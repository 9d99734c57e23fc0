"""Plain reference of rows in 8-bit integers -- TEST INFRASTRUCTURE.

Only ``tests/`` may import this module; the product never does, and this module imports nothing
from it.  A row's scale is max |x| / 127, 2^-126 at least; codes are rounded to nearest, ties to
even."""
from __future__ import annotations

import numpy as np


def padded(cols: int) -> int:
    return -(-cols // 128) * 128


def quantize_rows(x: np.ndarray):
    """(codes int8 [rows][padded(cols)], scales fp32 [rows]) of fp32 rows."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape
    codes = np.zeros((rows, padded(cols)), np.int8)
    with np.errstate(invalid="ignore"):
        most = np.abs(x).max(1) if rows else np.zeros(0, np.float32)
        good = np.isfinite(x).all(1)
        scale = np.maximum(most / np.float32(127), np.float32(2.0 ** -126)).astype(np.float32)
        codes[good, :cols] = np.rint(x[good] / scale[good, None]).astype(np.int8)
    scale[~good] = np.nan
    return codes, scale


def bf16(x: np.ndarray) -> np.ndarray:
    """fp32 values rounded to bfloat16 (nearest, ties to even), as fp32."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    with np.errstate(over="ignore"):
        r = ((u.astype(np.uint64) + 0x7fff + ((u >> 16) & 1)) & 0xffff0000).astype(np.uint32)
    out = r.view(np.float32).copy()
    out[np.isnan(x)] = np.nan
    return out
