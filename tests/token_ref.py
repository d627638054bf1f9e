"""Plain 64-bit implementations of the token operators (numpy), for their tests."""
from __future__ import annotations

import numpy as np

M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
LOW = 0xFFFFFFFF


def philox_scalar(counter, key, rounds=7):
    """Philox4x32 of one counter (4 words) and key (2 words), in Python integers."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = M0 * c[0], M1 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & LOW, (a >> 32) ^ c[3] ^ k[1], a & LOW]
        k = [(k[0] + W0) & LOW, (k[1] + W1) & LOW]
    return c


def keep(first, n, p, seed, call):
    """bool [n]: whether elements first .. first + n - 1 are kept."""
    thr = int(np.floor(float(np.float32(p)) * 65536.0 + 0.5))
    blk = np.arange(first // 8, (first + n + 7) // 8, dtype=np.uint64)
    u, sh = np.uint64, np.uint64(32)
    c = [blk & u(LOW), blk >> sh, np.full_like(blk, call & LOW),
         np.full_like(blk, (call >> 32) & LOW)]
    k = [seed & LOW, (seed >> 32) & LOW]
    for _ in range(7):
        a, b = c[0] * u(M0), c[2] * u(M1)
        c = [(b >> sh) ^ c[1] ^ u(k[0]), b & u(LOW), (a >> sh) ^ c[3] ^ u(k[1]), a & u(LOW)]
        k = [(k[0] + W0) & LOW, (k[1] + W1) & LOW]
    words = np.stack(c, 1)
    bits = np.stack([words & u(0xFFFF), words >> u(16)], 2).reshape(-1)
    at = first % 8
    return bits[at:at + n] >= thr


def drop(x, p, seed, call):
    """The dropped x in float64 (numbering the flat elements from 0)."""
    x = np.asarray(x, np.float64)
    thr = int(np.floor(float(np.float32(p)) * 65536.0 + 0.5))
    scale = 65536.0 / (65536 - thr) if thr < 65536 else 0.0
    k = keep(0, x.size, p, seed, call).reshape(x.shape)
    return np.where(k, np.where(k, x, 0.0) * scale, 0.0)


def embed_fwd(ids, table, scale, p, seed, call):
    out = np.zeros((ids.size, table.shape[1]))
    ok = (ids >= 0) & (ids < table.shape[0])
    out[ok] = np.asarray(table, np.float64)[ids[ok]] * scale
    return drop(out, p, seed, call)


def embed_bwd(ids, dout, V, scale, p, seed, call):
    """(dtable, per-element sum of |terms|, per-row count)."""
    g = drop(dout, p, seed, call) * scale
    ok = (ids >= 0) & (ids < V)
    d = np.zeros((V, dout.shape[1]))
    a = np.zeros_like(d)
    np.add.at(d, ids[ok], g[ok])
    np.add.at(a, ids[ok], np.abs(g[ok]))
    return d, a, np.bincount(ids[ok], minlength=V)


def xent(X, W, target, dloss):
    """dict of loss, lse, dX, dW and the magnitudes the error bounds need, over the rows with a
    target in [0, V)."""
    n, V = X.shape[0], W.shape[0]
    ok = (target >= 0) & (target < V)
    X, W = np.asarray(X, np.float64), np.asarray(W, np.float64)
    x, t, g = X[ok], target[ok], np.asarray(dloss, np.float64)[ok]
    r = {"loss": np.zeros(n), "lse": np.zeros(n), "dX": np.zeros(X.shape), "dW": np.zeros(W.shape),
         "absX": np.zeros(X.shape), "absW": np.zeros(W.shape), "allX": np.zeros(X.shape),
         "allW": np.zeros(W.shape), "zabs": 0.0}
    if not ok.any():
        return r
    z = x @ W.T
    top = z.max(1, keepdims=True)
    e = np.exp(z - top)
    lse = top[:, 0] + np.log(e.sum(1))
    r["lse"][ok] = lse
    r["loss"][ok] = lse - z[np.arange(len(t)), t]
    p = e / e.sum(1, keepdims=True)
    d = p.copy()
    d[np.arange(len(t)), t] -= 1.0
    d *= g[:, None]
    r["dX"][ok] = d @ W
    r["dW"] = d.T @ x
    # sums of |terms|, with the two parts of the target's term apart (p and 1 are rounded apart)
    m = p.copy()
    m[np.arange(len(t)), t] += 1.0
    m *= np.abs(g)[:, None]
    r["absX"][ok] = m @ np.abs(W)
    r["absW"] = m.T @ np.abs(x)
    # and of the terms with every probability 1 (and every weight the largest, for dW)
    r["allX"][ok] = np.abs(g)[:, None] * np.abs(W).sum(0)
    r["allW"][:] = np.abs(g).max() * np.abs(x).sum(0)
    r["zabs"] = float((np.abs(x) @ np.abs(W).T).max())
    return r
