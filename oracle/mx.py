"""MXFP4 in 64 bits, block by block: rounding, what codes stand for, and the two layouts.  Written from the definition of the
format and of the layouts; shares no code with the library."""
from __future__ import annotations

import math

import numpy as np

VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def round_value(v: float) -> int:
    """Code (0..15) of the nearest value; of two as near the one with the even code; 6 at most."""
    a = min(abs(v), 6.0)
    best = min(range(8), key=lambda c: (abs(VALUES[c] - a), c % 2))
    return best | (8 if math.copysign(1.0, v) < 0 else 0)


def round_block(x) -> tuple[list[int], int]:
    """Codes and scale byte of up to 32 values."""
    x = [float(v) for v in x]
    if not all(math.isfinite(v) for v in x):
        return [0] * len(x), 255
    m = max(abs(v) for v in x)
    e = max(-127, math.frexp(m)[1] - 1 - 2) if m else -127
    return [round_value(math.ldexp(v, -e)) for v in x], e + 127


def quantize(x: np.ndarray) -> tuple[np.ndarray, np.ndarray]:
    """codes uint8 [rows, cols] (one a value), scales uint8 [rows, cols/32]."""
    rows, cols = x.shape
    codes = np.zeros((rows, cols), np.uint8)
    scales = np.zeros((rows, cols // 32), np.uint8)
    for r in range(rows):
        for b in range(cols // 32):
            c, s = round_block(x[r, b * 32:(b + 1) * 32])
            codes[r, b * 32:(b + 1) * 32] = c
            scales[r, b] = s
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """float64 [rows, cols]; NaN where the scale byte is 255."""
    v = np.array(VALUES + tuple(-x for x in VALUES))[codes]
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(s, 32, axis=1)


def pack_rows(codes: np.ndarray, scales: np.ndarray) -> tuple[np.ndarray, np.ndarray]:
    """The bytes of the row layout."""
    rows, cols = codes.shape
    packed = codes[:, 0::2] | codes[:, 1::2] << 4
    filled = np.full((rows, -(-cols // 256) * 8), 127, np.uint8)
    filled[:, :cols // 32] = scales
    return packed, filled


def pack_tiles(codes: np.ndarray, scales: np.ndarray) -> tuple[np.ndarray, np.ndarray]:
    """The bytes of the tile layout, each put where the layout says."""
    rows, cols = codes.shape
    R, C, S = -(-rows // 32) * 32, -(-cols // 64) * 64, -(-cols // 256) * 256
    packed, _ = pack_rows(codes, scales)
    out = np.zeros(R * C // 2, np.uint8)
    out_s = np.full(R * S // 32, 127, np.uint8)
    for r in range(rows):
        for j in range(cols // 32):
            at = ((r // 32) * (C // 32) + j) * 512 + (r % 32) * 16
            out[at:at + 16] = packed[r, j * 16:(j + 1) * 16]
            out_s[((r // 32) * (S // 256) + j // 8) * 256 + (j % 2) * 128 + (r % 32) * 4 + j % 8 // 2] = scales[r, j]
    return out, out_s
