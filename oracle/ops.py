"""Plain numpy implementations, in 64 bits, of the operators beside the layer: routing from logits, rows to 8 bits, products of
8-bit codes, weighted sum of expert rows.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

SMALLEST = 2.0 ** -126


def scores(z, sigmoid):
    """[T, E] scores of logits; -inf and NaN score 0, several +inf share a softmax."""
    z = np.where(np.isnan(z), -np.inf, np.asarray(z, np.float64))
    if sigmoid:
        with np.errstate(over="ignore"):
            return 1 / (1 + np.exp(-z))
    top = z.max(axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        p = np.where(z == top, 1.0, np.exp(np.where(np.isfinite(z - top), z - top, -np.inf)))
    p[z == -np.inf] = 0
    total = p.sum(axis=1, keepdims=True)
    return np.divide(p, total, out=np.zeros_like(p), where=total > 0)


def route_scores(z, bias, k, *, sigmoid=False, n_groups=1, groups_kept=1, group_best=1, renorm=False, scale=1.0):
    """dict(ids, w [T, k], counts, offsets, perm, inv_perm)."""
    z = np.where(np.isnan(z), -np.inf, np.asarray(z, np.float64))
    T, E = z.shape
    s = scores(z, sigmoid)
    b = np.zeros(E) if bias is None else np.where(np.isnan(bias), -np.inf, np.asarray(bias, np.float64))
    ids = np.zeros((T, k), np.int64)
    for t in range(T):
        # without a bias the order of the logits, which is the order of the scores (64-bit scores meet at 1 and at 0)
        c = z[t] if bias is None and (n_groups == 1 or group_best == 1) else np.where(z[t] == -np.inf, -np.inf, s[t] + b)
        allowed = np.ones(E, bool)
        if n_groups > 1:
            best = -np.sort(-c.reshape(n_groups, -1), axis=1)[:, :group_best]
            value = np.where(best[:, -1] == -np.inf, best[:, -1] if group_best == 2 else best[:, 0], best.sum(axis=1))
            kept = sorted(range(n_groups), key=lambda g: (-value[g], g))[:groups_kept]
            allowed = np.repeat(np.isin(np.arange(n_groups), kept), E // n_groups)
        ids[t] = sorted(sorted(range(E), key=lambda e: (not allowed[e], -c[e], e))[:k])
    w = np.take_along_axis(s, ids, 1)
    if renorm:
        total = w.sum(axis=1, keepdims=True)
        w = np.divide(w, total, out=np.zeros_like(w), where=total > 0)
    flat = ids.reshape(-1)
    perm = np.argsort(flat, kind="stable")
    inv = np.empty(T * k, np.int64)
    inv[perm] = np.arange(T * k)
    counts = np.bincount(flat, minlength=E)
    return dict(ids=ids, w=w * scale, counts=counts, offsets=np.concatenate([[0], np.cumsum(counts)]), perm=perm, inv_perm=inv)


def quant_rows(x):
    """Codes (int64) and scales (float64 values of 32-bit numbers) of rows [rows, K]."""
    x = np.asarray(x, np.float64)
    bad = ~np.isfinite(x).all(axis=1)
    x = np.where(bad[:, None], 0.0, x)
    s = np.maximum((np.abs(x).max(axis=1) / 127).astype(np.float32).astype(np.float64), SMALLEST)
    return np.rint(x / s[:, None]).astype(np.int64), np.where(bad, np.nan, s)


def matmul_q8(q, s, w, ws, *, offsets=None, rows=None, swiglu=False):
    """q [R, K] codes with scales s [R]; w [G, N, K], ws [G, N] -> [M, N or N/2] float64, NaN where no group takes the row."""
    rows = np.arange(q.shape[0]) if rows is None else np.asarray(rows)
    offsets = [0, len(rows)] if offsets is None else offsets
    G, N, _ = w.shape
    y = np.full((len(rows), N), np.nan)
    for g in range(G):
        r = rows[offsets[g]:offsets[g + 1]]
        total = q[r].astype(np.float64) @ w[g].astype(np.float64).T      # whole numbers below 2^53: exact
        y[offsets[g]:offsets[g + 1]] = total * s[r][:, None] * np.asarray(ws[g], np.float64)
    if not swiglu:
        return y
    a, u = y[:, :N // 2], y[:, N // 2:]
    with np.errstate(over="ignore"):
        return a / (1 + np.exp(-a)) * u


def combine(y, w, inv_perm):
    T, k = w.shape
    return (np.asarray(w, np.float64)[:, :, None] * np.asarray(y, np.float64)[inv_perm].reshape(T, k, -1)).sum(axis=1)
