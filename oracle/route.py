"""The router of an MoE layer, the joining of its experts' outputs, and their
gradients, in fp64."""
from __future__ import annotations

import numpy as np


def _row(x):
    """(counts, lse, p) of one row of logits; a row with a NaN or +inf counts and is NaN."""
    if np.isnan(x).any() or (x == np.inf).any():
        return True, np.nan, np.full(len(x), np.nan)
    top = x.max()
    if top == -np.inf:
        return False, -np.inf, np.zeros(len(x))
    ex = np.exp(x - top)
    return True, top + np.log(ex.sum()), ex / ex.sum()


def route(logits, k, valid=None, renorm=True):
    x = np.asarray(logits, np.float64)
    T, E = x.shape
    experts = np.full((T, k), -1, np.int32)
    weights, lse, p = np.zeros((T, k)), np.full(T, -np.inf), np.zeros((T, E))
    n = 0
    for t in range(T):
        if valid is not None and not valid[t]:
            continue
        live, lse[t], p[t] = _row(x[t])
        n += live
        if not live:
            continue
        if np.isnan(lse[t]):
            weights[t] = np.nan
            continue
        order = sorted((e for e in range(E) if x[t, e] > -np.inf), key=lambda e: (-x[t, e], e))[:k]
        experts[t, :len(order)] = order
        weights[t, :len(order)] = p[t, order]
        if renorm:
            weights[t] /= weights[t].sum()
    bucket = np.where(experts < 0, E, experts).reshape(-1)
    counts = np.bincount(bucket, minlength=E + 1)[:E]
    order = np.argsort(bucket, kind="stable")
    slots = np.empty(T * k, np.int32)
    slots[order] = np.arange(T * k)
    z = lse[lse != -np.inf]
    losses = np.array([E / (k * n * n) * (counts * p.sum(0)).sum(), (z ** 2).sum() / n]) if n else np.zeros(2)
    return {"experts": experts, "weights": weights, "counts": np.r_[counts, n].astype(np.int32),
            "offsets": np.r_[0, np.cumsum(counts)].astype(np.int32), "rows": (order // k).astype(np.int32),
            "slots": slots.reshape(T, k), "lse": lse, "losses": losses}


def route_grad(logits, r, dweights=None, dlosses=None, renorm=True):
    """Gradient of the logits; r as ``route`` gave it."""
    x = np.asarray(logits, np.float64)
    T, E = x.shape
    k = r["experts"].shape[1]
    n = r["counts"][E]
    gb, gz = (0.0, 0.0) if dlosses is None else dlosses
    d = np.zeros((T, E))
    for t in range(T):
        if r["lse"][t] == -np.inf:
            continue
        p = _row(x[t])[2]
        a = E * r["counts"][:E] / (k * n * n)
        d[t] = gb * p * (a - (p * a).sum()) + gz * 2 / n * r["lse"][t] * p
        if dweights is None:
            continue
        S = [(e, j) for j, e in enumerate(r["experts"][t]) if e >= 0]
        up = np.zeros(E)
        for e, j in S:
            up[e] = dweights[t, j]
        q = np.zeros(E)
        chosen = [e for e, _ in S]
        q[chosen] = p[chosen]
        if renorm:
            if S:
                q /= q.sum()
            d[t] += q * (up - (q * up).sum())
        else:
            d[t] += p * up - p * (q * up).sum()
    return d


def combine(Z, slots, weights=None):
    w = np.ones(slots.shape) if weights is None else np.asarray(weights, np.float64)
    Y = np.zeros((len(slots), Z.shape[1]))
    for t in range(len(slots)):
        for j, s in enumerate(slots[t]):
            if 0 <= s < len(Z):
                Y[t] += w[t, j] * Z[s]
    return Y


def combine_grad(Z, slots, weights, dY):
    w = np.ones(slots.shape) if weights is None else np.asarray(weights, np.float64)
    dZ, dw = np.zeros(Z.shape), np.zeros(slots.shape)
    for t in range(len(slots)):
        for j, s in enumerate(slots[t]):
            if 0 <= s < len(Z):
                dZ[s] = w[t, j] * dY[t]
                dw[t, j] = dY[t] @ Z[s]
    return dZ, dw
