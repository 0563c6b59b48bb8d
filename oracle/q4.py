"""Weights in 4 bits with group scales, in fp64 numpy: the quantiser's definition,
the words' layout, and products. Test infrastructure only."""
from __future__ import annotations

import numpy as np


def row_words(ncols: int) -> int:
    return 4 * (-(-ncols // 32))


def _f32(v):
    return np.float64(np.float32(v))


def quantize(W, group: int, zeros: bool):
    """(codes uint8 [R, C], scale fp16 [R, G], zero uint8 [R, G] or None), group by
    group. Quotients are taken in fp64 and then rounded to fp32: for fp32 operands
    that is the correctly rounded fp32 quotient."""
    W = np.asarray(W, dtype=np.float64)
    R, C = W.shape
    G = -(-C // group)
    codes = np.zeros((R, C), np.uint8)
    scale = np.zeros((R, G), np.float16)
    zero = np.zeros((R, G), np.uint8) if zeros else None
    for r in range(R):
        for g in range(G):
            w = W[r, g * group:(g + 1) * group]
            if not np.all(np.isfinite(w)):
                scale[r, g] = np.nan
                continue
            lo, hi = min(0.0, w.min()), max(0.0, w.max())
            with np.errstate(over="ignore"):
                span = _f32(hi - lo) / 15.0 if zeros else np.abs(w).max() / 7.0
                s16 = np.float16(np.float32(min(_f32(span), 65504.0)))
            s = np.float64(s16)
            scale[r, g] = s16
            z = 8.0
            if zeros:
                z = min(max(np.rint(_f32(-lo / s)), 0.0), 15.0) if s > 0 else 0.0
                zero[r, g] = int(z)
            t = np.rint((w / s).astype(np.float32).astype(np.float64)) if s > 0 else np.zeros_like(w)
            codes[r, g * group:(g + 1) * group] = np.clip(t + z, 0, 15).astype(np.uint8)
    return codes, scale, zero


def pack(codes) -> np.ndarray:
    """uint32 words [R, row_words]: column c at bit 4 (c % 8) of word c / 8."""
    R, C = codes.shape
    out = np.zeros((R, row_words(C)), np.uint32)
    for c in range(C):
        out[:, c // 8] |= codes[:, c].astype(np.uint32) << np.uint32(4 * (c % 8))
    return out


def values(codes, scale, zero, group: int) -> np.ndarray:
    """s (u - z), exact in fp64."""
    of = np.arange(codes.shape[1]) // group
    z = 8.0 if zero is None else zero.astype(np.float64)[:, of]
    return (codes.astype(np.float64) - z) * scale.astype(np.float64)[:, of]
