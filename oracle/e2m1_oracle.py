"""Plain float64 oracle of the 4-bit rows (E2M1 in blocks of 32 with power-of-two scales).

TEST INFRASTRUCTURE ONLY, like ikv_oracle.py: it shares no code with the HIP library.
Pinned by tests/test_e2m1_oracle.py.
"""
from __future__ import annotations

import numpy as np

LEAST = 2.0 ** -100      # blocks are scaled as if their largest channel were at least this
MOST = 125               # exponent of the largest scale written
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def blocks(x):
    x = np.asarray(x, np.float64)
    return x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)


def scale_exponent(a: float) -> int:
    """The least e with 7 2^e >= a, at most MOST."""
    e = -110
    while 7.0 * 2.0 ** e < a and e < MOST:
        e += 1
    return e


def quantise(x):
    """Rows x [..., D] (exact float64 of their stored values) -> codes [..., D / 2], scale bytes [..., D / 32]."""
    x = blocks(x)
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0.0, x)
    a = np.maximum(np.abs(x).max(-1), LEAST)
    e = np.ceil(np.log2(a / 7.0)).astype(int)               # may be one off next to a power of two
    e = np.where(7.0 * np.exp2(e) < a, e + 1, e)
    e = np.where(7.0 * np.exp2(e - 1) >= a, e - 1, e)
    e = np.minimum(e, MOST)
    r = np.abs(x) / np.exp2(e)[..., None]
    down = np.clip(np.searchsorted(MAGNITUDES, r, side="right") - 1, 0, 7)      # MAGNITUDES[down] <= r
    up = np.minimum(down + 1, 7)
    lo, hi = r - MAGNITUDES[down], MAGNITUDES[up] - r
    code = np.where((hi < lo) | ((hi == lo) & (up % 2 == 0)), up, down)
    code = np.where(np.signbit(x), code | 8, code)
    code = np.where(bad[..., None], 0, code).astype(np.uint8)
    code = code.reshape(*code.shape[:-2], 32 * code.shape[-2])
    byte = np.where(bad, 255, e + 127).astype(np.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, byte


def values(codes, scales):
    """float64 rows [..., D] that codes [..., D / 2] with scale bytes [..., D / 32] stand for."""
    codes = np.asarray(codes, np.uint8)
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    v = np.where(c & 8, -1.0, 1.0) * MAGNITUDES[c & 7]
    s = np.asarray(scales, np.int64)
    s = np.where(s == 255, np.nan, np.exp2(s.astype(np.float64) - 127))
    return (blocks(v) * s[..., None]).reshape(v.shape)
