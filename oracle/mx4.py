"""Microscaled 4-bit floats in fp64 numpy: the quantiser's definition and the values of
codes. The words' layout is that of ``oracle.q4.pack``. Test infrastructure only."""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def nearest(t: float) -> int:
    """The code 0 .. 7 nearest to t >= 0, of two as near the even one."""
    d = np.abs(MAGNITUDES - t)
    return min(range(8), key=lambda c: (d[c], c % 2))


def quantize(W):
    """(codes uint8 [R, C], scale uint8 [R, blocks]), block by block."""
    W = np.asarray(W, dtype=np.float64)
    R, C = W.shape
    codes = np.zeros((R, C), np.uint8)
    scale = np.zeros((R, -(-C // 32)), np.uint8)
    for r in range(R):
        for b in range(scale.shape[1]):
            w = W[r, 32 * b:32 * b + 32]
            if not np.all(np.isfinite(w)):
                scale[r, b] = 255
                continue
            m = np.abs(w).max()
            e = max(int(np.frexp(m)[1]) - 1 - 2, -127) if m > 0 else -127
            scale[r, b] = e + 127
            for i, v in enumerate(w):
                codes[r, 32 * b + i] = nearest(abs(v) * 2.0 ** -e) | (8 if np.signbit(v) else 0)
    return codes, scale


def values(codes, scale) -> np.ndarray:
    """v 2^(e - 127), exact in fp64; NaN where e is 255."""
    of = np.arange(codes.shape[1]) // 32
    v = MAGNITUDES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    e = scale.astype(np.int64)
    return v * np.where(e == 255, np.nan, np.ldexp(1.0, e - 127))[:, of]
