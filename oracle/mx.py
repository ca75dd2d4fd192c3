"""Rows in microscaled 4-bit floating point (OCP Microscaling Formats v1.0, MXFP4), in 64 bits and numpy.

TEST INFRASTRUCTURE ONLY, written from the format's definition: a code is a sign and one of eight magnitudes (E2M1), a block of 32 of
them has a power of two (E8M0, 2^(byte - 127); 255: NaN).
"""
from __future__ import annotations

from typing import Tuple

import numpy as np

BLOCK = 32
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def dequantize(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """codes uint8 [..., inner / 2], scales uint8 [..., inner / 32] -> float64 [..., inner]"""
    nibbles = np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:-1], -1)
    values = np.where(nibbles & 8, -1.0, 1.0) * MAGNITUDES[nibbles & 7]
    factor = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return values * np.repeat(factor, BLOCK, axis=-1)


def quantize(x: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """float [..., inner] -> (codes, scales).  Every magnitude is compared with all eight that a code has: the nearest one, of two
    that are equally near the even code.  The sign of an element stays, a zero's too."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK)
    top = np.abs(blocks).max(axis=-1)
    finite = np.isfinite(blocks).all(axis=-1)
    exponent = np.where(finite & (top > 0), np.frexp(np.where(finite, top, 1.0))[1] - 1, -1000)  # floor(log2(top))
    scales = np.where(finite, np.maximum(exponent - 2, -127) + 127, 255).astype(np.uint8)
    unit = np.ldexp(1.0, scales.astype(np.int64) - 127)[..., None]
    y = np.where(finite[..., None], np.abs(blocks) / unit, 0.0)
    code, best = np.zeros(y.shape, dtype=np.uint8), np.full(y.shape, np.inf)
    for c in (0, 2, 4, 6, 1, 3, 5, 7):  # (an odd code has to be nearer)
        nearer = np.abs(y - MAGNITUDES[c]) < best
        best = np.where(nearer, np.abs(y - MAGNITUDES[c]), best)
        code = np.where(nearer, c, code).astype(np.uint8)
    code = (code | np.where(np.signbit(blocks) & finite[..., None], 8, 0)).astype(np.uint8)
    code = code.reshape(x.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4).astype(np.uint8), scales
