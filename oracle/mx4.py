"""Microscaled 4-bit floats and the experts' products on them, in fp64.

A block of 32 entries has one scale 2^(s - 127), s - 127 = floor(log2 max) - 2
(at least -127, and 0 stands for a block of zeros), and every entry is the
nearest of +-{0, 1/2, 1, 3/2, 2, 3, 4, 6} scales, ties to the even code.  A
block with a NaN or an infinity has s = 255 and codes 0 and stands for NaN.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
BLOCK = 32


def quantize(X):
    """Codes uint8 [..][cols/2] (entry 2i in the low half of byte i) and scales
    uint8 [..][cols/32] of rows X."""
    X = np.asarray(X, np.float64)
    B = X.reshape(*X.shape[:-1], -1, BLOCK)
    lost = ~np.isfinite(B).all(-1)
    A = np.where(np.isfinite(B), np.abs(B), 0.0)
    top = A.max(-1)
    e = np.where(top > 0, np.frexp(top)[1] - 1 - 2, -127)  # frexp: top = m 2^x, m in [1/2, 1)
    e = np.maximum(e, -127)
    m = A / np.ldexp(1.0, e)[..., None]
    # nearest grid value; half way between two (above one midpoint fewer than at or above), the even code
    mid = (GRID[1:] + GRID[:-1]) / 2
    low, high = np.searchsorted(mid, m, "left"), np.searchsorted(mid, m, "right")
    code = np.where(low % 2 == 0, low, high).astype(np.uint8)
    code |= np.signbit(B).astype(np.uint8) << 3
    code = np.where(lost[..., None], 0, code).astype(np.uint8).reshape(X.shape)
    scales = np.where(lost, 255, e + 127).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scales


def dequantize(codes, scales):
    """fp64 values of MX4 rows."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = GRID[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(s, BLOCK, axis=-1)


def silu(v):
    with np.errstate(over="ignore"):
        return v / (1 + np.exp(-v))


def product(W, X, offsets=None, rows=None, S=None, glu=False):
    """y_s = W_e x_{rows[s]} for slots in expert order; W [E][N][K] and X in fp64."""
    E = W.shape[0]
    S = (len(X) if rows is None else len(rows)) if S is None else S
    offsets = np.array([0, S]) if offsets is None else offsets
    Y = np.zeros((S, W.shape[1]))
    for e in range(E):
        slots = np.arange(max(0, offsets[e]), min(S, offsets[e + 1]))
        r = slots if rows is None else rows[slots]
        there = (r >= 0) & (r < len(X))
        Y[slots[there]] = X[r[there]] @ W[e].T
    if glu:
        N = W.shape[1] // 2
        Y = silu(Y[:, :N]) * Y[:, N:]
    return Y


def product_grad(W, dY, offsets=None):
    """dx_s = W_e^T dy_s."""
    return product(np.swapaxes(W, 1, 2), dY, offsets)
