"""Plain implementations of the operators that answer with a vocabulary (numpy), for their tests: logits
and distillation in 64 bits, adjusted logits in 32 bits, operation by operation, as their definition says."""
from __future__ import annotations

import numpy as np


def pack_mask(allowed):
    """int32 [masks, ceil(V / 32)]: bit v % 32 of word v / 32 of allowed [masks, V]."""
    G, V = allowed.shape
    bits = np.zeros((G, (V + 31) // 32 * 32), np.uint8)
    bits[:, :V] = allowed
    return np.packbits(bits, axis=1, bitorder="little").view("<u4").astype(np.uint32).view(np.int32)


def adjusted(z, bias=None, allowed=None, mask_row=None, history=None, penalty=None):
    """fp32 [n, V]; history: a list of tokens a row; allowed bool [masks, V]."""
    z = np.asarray(z, np.float32).copy()
    n, V = z.shape
    with np.errstate(all="ignore"):
        if bias is not None:
            z = z + np.asarray(bias, np.float32)[None]
        if history is not None:
            for i, ids in enumerate(history):
                ids = np.asarray(ids, np.int64)
                ids = ids[(ids >= 0) & (ids < V)]
                v, c = np.unique(ids, return_counts=True)
                rep, presence, frequency = (np.float32(p) for p in penalty[i])
                at = z[i, v]
                at = np.where(at > 0, at / rep, at * rep).astype(np.float32)
                z[i, v] = at - (presence + frequency * c.astype(np.float32)).astype(np.float32)
        if allowed is not None:
            G = allowed.shape[0]
            if mask_row is None:
                mask_row = np.zeros(n, np.int64) if G == 1 else np.arange(n)
            for i, g in enumerate(mask_row):
                if 0 <= g < G:
                    z[i, ~allowed[g]] = -np.inf
    return z


def top(z, K):
    """(values, ids, lse) of fp32 rows: falling, equal values by rising id; -inf and NaN are no answers."""
    n, V = z.shape
    vals, ids = np.full((n, K), -np.inf, np.float32), np.full((n, K), -1, np.int32)
    lse = np.full(n, -np.inf)
    for i in range(n):
        ok = np.flatnonzero(z[i] > -np.inf)
        order = ok[np.argsort(-z[i, ok].astype(np.float64), kind="stable")][:K]
        vals[i, :len(order)], ids[i, :len(order)] = z[i, order], order
        if np.isnan(z[i]).any() or np.isposinf(z[i]).any():
            lse[i] = np.nan
        elif len(ok):
            m = float(z[i, ok].max())
            lse[i] = m + np.log(np.exp(z[i, ok].astype(np.float64) - m).sum())
    return vals, ids, lse


def distill(X, W, ids, logits, tau, g):
    """dict of loss, lse, dX, dW and the magnitudes the error bounds need."""
    n, V = X.shape[0], W.shape[0]
    X, W = np.asarray(X, np.float64), np.asarray(W, np.float64)
    ok = (ids >= 0) & (ids < V) & (logits > -np.inf)
    rows = ok.any(1)
    r = {"loss": np.zeros(n), "lse": np.zeros(n), "dX": np.zeros(X.shape), "dW": np.zeros(W.shape),
         "absX": np.zeros(X.shape), "absW": np.zeros(W.shape), "allX": np.zeros(X.shape),
         "allW": np.zeros(W.shape), "zabs": 0.0, "rows": rows}
    if not rows.any():
        return r
    x, t, m, gg = X[rows], np.where(ok, ids, 0)[rows], ok[rows], np.asarray(g, np.float64)[rows] * tau
    u = np.where(m, np.asarray(logits, np.float64)[rows] / tau, -np.inf)
    e = np.exp(u - u.max(1, keepdims=True))
    q = e / e.sum(1, keepdims=True)
    log_q = np.where(m, u - u.max(1, keepdims=True) - np.log(e.sum(1, keepdims=True)), 0.0)
    z = x @ W.T / tau
    top = z.max(1, keepdims=True)
    p = np.exp(z - top)
    r["lse"][rows] = lse = top[:, 0] + np.log(p.sum(1))
    p /= p.sum(1, keepdims=True)
    zk = np.take_along_axis(z, t, 1)
    r["loss"][rows] = tau * tau * (np.where(m, q * (log_q - zk), 0.0).sum(1) + lse)
    Q = np.zeros_like(p)
    np.add.at(Q, (np.arange(len(t))[:, None], t), np.where(m, q, 0.0))
    r["dX"][rows] = (gg[:, None] * (p - Q)) @ W
    r["dW"] = (gg[:, None] * (p - Q)).T @ x
    r["absX"][rows] = (np.abs(gg)[:, None] * (p + Q)) @ np.abs(W)
    r["absW"] = (np.abs(gg)[:, None] * (p + Q)).T @ np.abs(x)
    r["allX"][rows] = np.abs(gg)[:, None] * np.abs(W).sum(0)
    r["allW"][:] = np.abs(gg).max() * np.abs(x).sum(0)
    r["zabs"] = float((np.abs(x) @ np.abs(W).T).max()) / tau
    r["uabs"] = float(np.abs(np.where(m, u, 0.0)).max())
    return r
