"""What a cache held in 4 bits stands for, in float64.

Test infrastructure only (see the package docstring).

A row x of one token and head becomes low = min x, scale = fp16((max x - low) /
15) with the quotient in float32, and the codes nearest to (x - low) / scale,
ties to even, 0..15; it stands for low + scale * code. A row with a non-finite
element stands for NaN throughout.
"""
from __future__ import annotations

import numpy as np


def kv4_quantise(x):
    """fp16 rows [..., d] -> codes [..., d] (uint8), scale and low [..., 1]."""
    x = np.asarray(x)
    assert x.dtype == np.float16
    bad = ~np.isfinite(x).all(axis=-1, keepdims=True)
    y = np.where(bad, np.float16(0), x).astype(np.float64)
    low = y.min(axis=-1, keepdims=True)
    scale = ((y.max(axis=-1, keepdims=True) - low).astype(np.float32) / np.float32(15)).astype(np.float16)
    s = scale.astype(np.float64)
    code = np.zeros_like(y)
    np.divide(y - low, s, out=code, where=s > 0)
    code = np.clip(np.rint(code), 0, 15).astype(np.uint8)
    nan = np.float16(np.nan)
    return code, np.where(bad, nan, scale), np.where(bad, nan, low.astype(np.float16))


def kv4_values(x):
    """The values fp16 rows stand for once stored, float64."""
    code, scale, low = kv4_quantise(np.asarray(x, np.float16))
    return code * scale.astype(np.float64) + low.astype(np.float64)
