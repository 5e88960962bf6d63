"""Plain float64 oracle of the 8-bit cache and of the attention with a window and sinks.

TEST INFRASTRUCTURE ONLY, like ikv_oracle.py: it shares no code with the HIP library.
Pinned by tests/test_quant_oracle.py (hand-worked rows, ties, the E4M3 value table, closed
forms of the attention).
"""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

LEAST = 2.0 ** -100      # rows are scaled as if their largest channel were at least this


def e4m3_values() -> np.ndarray:
    """The 127 non-negative finite E4M3 values; their index is their code."""
    return np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])


def quantise(x, code: str):
    """Rows x [..., D] (exact float64 of their stored values) -> (codes as bytes [..., D], scale float32 [...])."""
    x = np.asarray(x, np.float64)
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0.0, x)
    a = np.maximum(np.abs(x).max(-1), LEAST)
    if code == "int8":
        codes = np.rint(127.0 * x / a[..., None]).astype(np.int8).view(np.uint8)
        scale = (a / 127.0).astype(np.float32)
    else:
        e = np.ceil(np.log2(a) - math.log2(448.0)).astype(int)
        e = np.where(448.0 * np.exp2(e) < a, e + 1, e)
        e = np.where(448.0 * np.exp2(e - 1) >= a, e - 1, e)
        s = np.exp2(e)
        r = np.abs(x) / s[..., None]
        v = e4m3_values()
        hi = np.searchsorted(v, r)                       # v[hi - 1] < r <= v[hi]
        lo = np.maximum(hi - 1, 0)
        down, up = r - v[lo], v[hi] - r
        idx = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
        codes = (idx | np.where(np.signbit(x), 128, 0)).astype(np.uint8)
        scale = s.astype(np.float32)
    return np.where(bad[..., None], 0, codes).astype(np.uint8), np.where(bad, np.float32(np.nan), scale).astype(np.float32)


def int8_code(x: float, a: float) -> int:
    """The int8 code of one channel by exact rational arithmetic."""
    r = Fraction(127) * Fraction(x) / Fraction(max(a, LEAST))
    f = math.floor(r)
    d = r - f
    return f if d < Fraction(1, 2) or (d == Fraction(1, 2) and f % 2 == 0) else f + 1


def code_values(codes, code: str) -> np.ndarray:
    """float64 values of code bytes."""
    c = np.asarray(codes, np.uint8)
    if code == "int8":
        return c.view(np.int8).astype(np.float64)
    v = np.append(e4m3_values(), np.nan)[c & 127]
    return np.where(c & 128, -v, v)


def seen(N: int, n: int, sinks: int, window: int) -> np.ndarray:
    """[n, N] truth values: what token t of the newest n of N list entries sees."""
    i = (N - n + np.arange(n))[:, None]
    j = np.arange(N)[None]
    ok = j <= i
    return ok & ((j < sinks) | (j > i - window)) if window else ok


def attend(q, k, v, sinks: int = 0, window: int = 0):
    """Attention of one layer: q [Hq, n, D], rows of the list k, v [N, Hkv, D] (float64).

    Returns (out [Hq, n, D], spread [Hq, n, D], reach [Hq, n]): spread is sum_j w_j |v_j|, reach the
    largest sum_d |q_d k_jd| / sqrt(D) of an entry seen; error bounds are stated in them."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    Hq, n, D = q.shape
    N, Hkv = k.shape[:2]
    out, spread, reach = np.zeros_like(q), np.zeros_like(q), np.zeros((Hq, n))
    ok = seen(N, n, sinks, window)
    for h in range(Hq):
        g = h // (Hq // Hkv)
        for t in range(n):
            j = np.nonzero(ok[t])[0]
            if len(j) == 0:
                continue
            x = k[j, g] @ q[h, t] / math.sqrt(D)
            w = np.exp(x - x.max())
            w /= w.sum()
            out[h, t] = w @ v[j, g]
            spread[h, t] = w @ np.abs(v[j, g])
            reach[h, t] = (np.abs(k[j, g]) @ np.abs(q[h, t])).max() / math.sqrt(D)
    return out, spread, reach
