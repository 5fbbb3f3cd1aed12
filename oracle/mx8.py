"""Microscaled 8-bit floats, and silu(gate) * up with its gradient at values
kept in them, in fp64.

A block of 32 entries has one scale 2^(s - 127), the smallest power of two (at
least 2^-127) at which the block's largest magnitude does not pass 448, and
every entry is the nearest E4M3 float (ties to even) of its quotient by the
scale.  A block with a NaN or an infinity has s = 255 and codes 0 and stands for
NaN.
"""
from __future__ import annotations

import numpy as np

from .mx4 import silu

BLOCK = 32
# the magnitudes of codes 0 .. 126: eighths below 2^-6, then eight steps to every power of two
GRID = np.array([np.ldexp(c, -9) if c < 8 else np.ldexp(8 + c % 8, c // 8 - 10) for c in range(127)])


def quantize(X):
    """Codes uint8 [..][cols] and scales uint8 [..][cols/32] of rows X."""
    X = np.asarray(X, np.float64)
    B = X.reshape(*X.shape[:-1], -1, BLOCK)
    lost = ~np.isfinite(B).all(-1)
    A = np.where(np.isfinite(B), np.abs(B), 0.0)
    top = A.max(-1)
    e = np.where(top > 0, np.frexp(top)[1] - 1 - 8, -127)  # top in [2^8, 2^9) scales
    e = np.where(top > np.ldexp(448.0, e), e + 1, e)
    e = np.maximum(e, -127)
    m = A / np.ldexp(1.0, e)[..., None]
    mid = (GRID[1:] + GRID[:-1]) / 2
    low, high = np.searchsorted(mid, m, "left"), np.searchsorted(mid, m, "right")
    code = np.where(low % 2 == 0, low, high).astype(np.uint8)
    code |= np.signbit(B).astype(np.uint8) << 7
    code = np.where(lost[..., None], 0, code).astype(np.uint8).reshape(X.shape)
    return code, np.where(lost, 255, e + 127).astype(np.uint8)


def dequantize(codes, scales):
    """fp64 values of MX8 rows."""
    grid = np.append(GRID, np.nan)  # (code 127 stands for no number)
    v = grid[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(s, BLOCK, axis=-1)


def glu(GU):
    """silu(g) * u of rows [g, u]."""
    N = GU.shape[1] // 2
    return silu(GU[:, :N]) * GU[:, N:]


def glu_grad(GU, dH):
    """Gradient of ``glu`` at GU."""
    N = GU.shape[1] // 2
    g, u = GU[:, :N], GU[:, N:]
    with np.errstate(over="ignore"):
        s = 1 / (1 + np.exp(-g))
    return np.concatenate((dH * u * s * (1 + g * (1 - s)), dH * g * s), 1)
