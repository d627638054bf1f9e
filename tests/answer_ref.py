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
