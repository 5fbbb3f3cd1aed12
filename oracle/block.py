"""The norm before an MoE layer, and the gradient of its experts' weights, in
fp64 (the experts' products themselves: ``mx4.product`` and
``mx4.product_grad``, which take any weights)."""
from __future__ import annotations

import numpy as np


def rms_norm(v, w, eps):
    """(y, inv) of rows v."""
    v = np.asarray(v, np.float64)
    inv = 1 / np.sqrt((v * v).mean(1) + eps)
    return v * inv[:, None] * w, inv


def rms_norm_grad(v, w, inv, dy, dsum=None):
    """(dx, dw) from the gradient of y and of v itself."""
    n = v * inv[:, None]
    g = dy * w
    dx = inv[:, None] * (g - n * (g * n).mean(1, keepdims=True))
    return (dx if dsum is None else dx + dsum), (dy * n).sum(0)


def weight_grad(dY, X, E=1, offsets=None, rows=None):
    """dW_e = sum over e's slots of dy_s x_{rows[s]}^T."""
    S = len(dY)
    offsets = np.array([0, S]) if offsets is None else offsets
    dW = np.zeros((E, dY.shape[1], X.shape[1]))
    for e in range(E):
        for s in range(max(0, offsets[e]), min(S, offsets[e + 1])):
            r = s if rows is None else rows[s]
            if 0 <= r < len(X):
                dW[e] += np.outer(dY[s], X[r])
    return dW
