"""Cases of the token operators at the two ends of a GGNN: the embedding lookup that makes the
initial node states, dropout, and the softmax cross entropy of node states against a vocabulary,
each forward and with its gradient.

`listed()` / `draw()` give cases, `prepare()` a case's inputs, `run()` one pass (the library's calls
where `own` is true, elementary torch operations in 32 bits where it is not), `exact()` the same
outputs in 64 bits and `work()` the bytes and operations a pass cannot do without.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# --------------------------------------------------------------------------------------- cases


def listed():
    return [
        # initial states of the 512-node graph of the correctness workload: all latency
        dict(name="embed_fwd_512", op="embed_fwd", n=512, H=64, V=1000, dtype="f32", p=0.0),
        # initial states of the largest supergraph at the widest state, embedding dropout on
        dict(name="embed_fwd_131k", op="embed_fwd", n=131072, H=256, V=49999, dtype="bf16", p=0.1),
        # table gradient of one 20k-node graph
        dict(name="embed_bwd_20k", op="embed_bwd", n=20001, H=128, V=10000, p=0.1),
        # table gradient of the largest supergraph at the widest state
        dict(name="embed_bwd_131k", op="embed_bwd", n=131071, H=256, V=49999, p=0.0),
        # dropout of one small graph's states, an odd number of elements
        dict(name="dropout_fwd_33k", op="dropout_fwd", n=32767, dtype="f32", p=0.5, residual=False),
        # dropout of a GGNN layer's output added to its input (131072 x 256 states)
        dict(name="dropout_fwd_34M", op="dropout_fwd", n=33554432, dtype="bf16", p=0.1,
             residual=True),
        # gradient through dropout at the training step's size (100003 x 256 states)
        dict(name="dropout_bwd_26M", op="dropout_bwd", n=25600768, p=0.1),
        # one node scored against the whole vocabulary: a completion request
        dict(name="xent_score_1", op="xent_fwd", n=1, H=128, V=32000, dtype="bf16", labelled=1.0),
        # the correctness workload's graph, all of it in 32 bits
        dict(name="xent_train_512", op="xent_train", n=512, H=64, V=4001, dtype="f32", grad="f32",
             labelled=1.0),
        # one 20k-node graph in 32 bits
        dict(name="xent_train_f32_20k", op="xent_train", n=20000, H=128, V=32000, dtype="f32",
             grad="f32", labelled=1.0),
        # a packed batch of which 15% of the nodes are masked out and to be predicted
        dict(name="xent_train_masked_72k", op="xent_train", n=71969, H=64, V=10000, dtype="bf16",
             grad="f32", labelled=0.15),
        # every node of half the largest supergraph labelled, widest state, largest vocabulary
        dict(name="xent_train_65k", op="xent_train", n=65537, H=256, V=49999, dtype="bf16",
             grad="bf16", labelled=1.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "dropout_fwd", "dropout_bwd", "xent_fwd",
                     "xent_train", "xent_train"])
    H = 32 * rng.randint(1, 8)
    p = rng.choice([0.0, 0.1, 0.25, 0.5])
    if op == "embed_fwd":
        return dict(op=op, n=_log_int(rng, 1, 131072), H=H, V=_log_int(rng, 2, 49999),
                    dtype=rng.choice(["f32", "bf16"]), p=p)
    if op == "embed_bwd":
        return dict(op=op, n=_log_int(rng, 1, 131071), H=H, V=_log_int(rng, 2, 49999), p=p)
    if op == "dropout_fwd":
        return dict(op=op, n=_log_int(rng, 1000, 33554432), dtype=rng.choice(["f32", "bf16"]), p=p,
                    residual=rng.random() < 0.5)
    if op == "dropout_bwd":
        return dict(op=op, n=_log_int(rng, 1000, 25600768), p=p)
    case = dict(op=op, n=_log_int(rng, 1, 65537), H=H, V=_log_int(rng, 2, 49999),
                dtype=rng.choice(["f32", "bf16"]), labelled=rng.choice([0.15, 0.5, 1.0]))
    if op == "xent_train":
        case["grad"] = "f32" if case["dtype"] == "f32" else rng.choice(["f32", "bf16"])
    # 32-bit inputs stay within a quarter of the largest case's products
    most = 65537 * 49999 * 256 // (4 if case["dtype"] == "f32" else 1)
    while case["n"] * case["V"] * H > most:
        case["n"] = (case["n"] + 1) // 2
    return case


# --------------------------------------------------------------------------------------- inputs


def _labelled(case):
    return max(1, int(round(case["labelled"] * case["n"])))


def _zipf(n, V, gen):
    """n ids in [0, V), id r drawn with weight 1 / (r + 2): token frequencies, in falling order."""
    w = 1.0 / torch.arange(2, V + 2, device="cuda", dtype=torch.float64)
    cdf = torch.cumsum(w, 0)
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) * cdf[-1]
    return torch.searchsorted(cdf, u).clamp_(max=V - 1).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    s = dict(case)
    # the counters of the dropout masks, as a training loop hands them over: a run's seed and the
    # number of the call
    s["seed"] = (seed * 0x9E3779B97F4A7C15 + 0x1906) & 0x7FFFFFFFFFFFFFFF
    s["call"] = 11786 + seed % 1000
    op, n = case["op"], case["n"]
    if op in ("embed_fwd", "embed_bwd"):
        H, V = case["H"], case["V"]
        ids = _zipf(n, V, gen)
        # the rows that fill a supergraph up to whole blocks hold no node
        ids[n - n // 50:] = -1
        s["ids"] = ids
        s["scale"] = math.sqrt(H)
        if op == "embed_fwd":
            s["table"] = (normal(V, H) / math.sqrt(H)).to(DTYPES[case["dtype"]])
        else:
            s["dout"] = normal(n, H) * 1e-3
    elif op == "dropout_fwd":
        s["x"] = normal(n).to(DTYPES[case["dtype"]])
        s["res"] = normal(n).to(DTYPES[case["dtype"]]) if case["residual"] else None
    elif op == "dropout_bwd":
        s["dy"] = normal(n) * 1e-3
    else:
        H, V = case["H"], case["V"]
        target = _zipf(n, V, gen)
        W = (normal(V, H) * (2.0 / math.sqrt(H))).to(DTYPES[case["dtype"]])
        # states that have learnt something about their targets
        lean = 2.0 * torch.rand(n, 1, generator=gen, device="cuda")
        s["X"] = (normal(n, H) + lean * W.float()[target.long()]).to(DTYPES[case["dtype"]])
        m = _labelled(case)
        order = torch.rand(n, generator=gen, device="cuda").argsort()
        target[order[m:]] = -1
        s["W"], s["target"] = W, target
        if op == "xent_train":
            # the mean over the labelled nodes, each with a weight of its own
            s["dloss"] = (0.5 + torch.rand(n, generator=gen, device="cuda")) / m
    return s


# --------------------------------------------------------------------------------------- plain form

_M0, _M1, _K0, _K1, _LOW = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85, 0xFFFFFFFF


def _threshold(p):
    return int(math.floor(float(np.float32(p)) * 65536.0 + 0.5))


def _keep(n, p, seed, call):
    """Truth value of each of n elements: Philox4x32 with 7 rounds, key = seed, counter =
    (element / 8, call); element i has the 16 bits from 16 (i % 2) on of word (i % 8) / 2 and is
    kept where they are p * 65536 or more."""
    i = torch.arange((n + 7) // 8, device="cuda", dtype=torch.int64)
    c0, c1 = i & _LOW, i >> 32
    c2 = torch.full_like(i, call & _LOW)
    c3 = torch.full_like(i, (call >> 32) & _LOW)
    k0, k1 = seed & _LOW, (seed >> 32) & _LOW
    c0, c1, c2, c3 = _rounds(c0, c1, c2, c3, k0, k1, 7)
    words = torch.stack([c0, c1, c2, c3], 1)
    halves = torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)[:n]
    return halves >= _threshold(p)


def _rounds(c0, c1, c2, c3, k0, k1, left):
    if not left:
        return c0, c1, c2, c3
    a, b = c0 * _M0, c2 * _M1
    return _rounds(((b >> 32) & _LOW) ^ c1 ^ k0, b & _LOW, ((a >> 32) & _LOW) ^ c3 ^ k1, a & _LOW,
                   (k0 + _K0) & _LOW, (k1 + _K1) & _LOW, left - 1)


def _scale_kept(p):
    t = _threshold(p)
    return 65536.0 / (65536 - t) if t < 65536 else 0.0


def _drop(x, s):
    if s["p"] == 0.0:
        return x
    keep = _keep(x.numel(), s["p"], s["seed"], s["call"]).view(x.shape)
    return torch.where(keep, x * _scale_kept(s["p"]), torch.zeros_like(x))


def _plain(s):
    op = s["op"]
    if op == "embed_fwd":
        ids = s["ids"].long()
        rows = s["table"].float()[ids.clamp(min=0)] * s["scale"]
        rows = torch.where((ids >= 0)[:, None], rows, torch.zeros_like(rows))
        return _drop(rows, s).to(s["table"].dtype)
    if op == "embed_bwd":
        ids = s["ids"].long()
        g = _drop(s["dout"], s) * s["scale"]
        g = torch.where((ids >= 0)[:, None], g, torch.zeros_like(g))
        d = torch.zeros(s["V"], s["H"], device="cuda")
        return d.index_add_(0, ids.clamp(min=0), g)
    if op == "dropout_fwd":
        y = _drop(s["x"].float(), s)
        return (y if s["res"] is None else y + s["res"].float()).to(s["x"].dtype)
    if op == "dropout_bwd":
        return _drop(s["dy"], s).clone()
    target = s["target"].long()
    valid = target >= 0
    X, W = s["X"].float(), s["W"].float()
    X = torch.where(valid[:, None], X, torch.zeros_like(X))
    logits = X @ W.t()
    top = logits.amax(1)
    probs = torch.exp(logits - top[:, None])
    total = probs.sum(1)
    lse = torch.where(valid, top + torch.log(total), torch.zeros_like(top))
    at = target.clamp(min=0)[:, None]
    loss = torch.where(valid, lse - logits.gather(1, at)[:, 0], torch.zeros_like(lse))
    if op == "xent_fwd":
        return loss, lse
    g = torch.where(valid, s["dloss"], torch.zeros_like(lse))
    probs *= (g / total)[:, None]
    probs.scatter_add_(1, at, -g[:, None])
    out = DTYPES[s["grad"]]
    return loss, lse, (probs @ W).to(out), (probs.t() @ X).to(out)


# ------------------------------------------------------------------------------ the library


def _own(s):
    from paper_1906_11786_gb300 import lib as L

    op = s["op"]
    if op == "embed_fwd":
        if "out" not in s:
            s["out"] = torch.empty(s["n"], s["H"], device="cuda", dtype=s["table"].dtype)
        L.embed_fwd(s["dtype"], s["ids"], s["table"], s["out"], scale=s["scale"], p=s["p"],
                    seed=s["seed"], call=s["call"])
        return s["out"]
    if op == "embed_bwd":
        if "out" not in s:
            s["out"] = torch.empty(s["V"], s["H"], device="cuda")
            s["ws"] = torch.empty(L.embed_workspace_bytes(s["n"], s["H"], s["V"]), device="cuda",
                                  dtype=torch.uint8)
        L.embed_bwd(s["ids"], s["dout"], s["out"], s["ws"], scale=s["scale"], p=s["p"],
                    seed=s["seed"], call=s["call"])
        return s["out"]
    if op == "dropout_fwd":
        if "out" not in s:
            s["out"] = torch.empty_like(s["x"])
        L.dropout_fwd(s["dtype"], s["x"], s["out"], s["p"], s["seed"], s["call"], residual=s["res"])
        return s["out"]
    if op == "dropout_bwd":
        if "out" not in s:
            s["out"] = torch.empty_like(s["dy"])
        L.dropout_bwd(s["dy"], s["out"], s["p"], s["seed"], s["call"])
        return s["out"]
    n, H, V = s["n"], s["H"], s["V"]
    if "loss" not in s:
        s["loss"] = torch.empty(n, device="cuda")
        s["lse"] = torch.empty(n, device="cuda")
        need = L.xent_workspace_bytes(s["dtype"], n, H, V, L.BG_OP_XENT_FWD)
        if op == "xent_train":
            s["dX"] = torch.empty(n, H, device="cuda", dtype=DTYPES[s["grad"]])
            s["dW"] = torch.empty(V, H, device="cuda", dtype=DTYPES[s["grad"]])
            need = max(need, L.xent_workspace_bytes(s["dtype"], n, H, V, L.BG_OP_XENT_BWD))
        s["ws"] = torch.empty(need, device="cuda", dtype=torch.uint8)
    L.xent_fwd(s["dtype"], s["X"], s["W"], s["target"], s["loss"], s["lse"], s["ws"])
    if op == "xent_fwd":
        return s["loss"], s["lse"]
    L.xent_bwd(s["dtype"], s["X"], s["W"], s["target"], s["lse"], s["dloss"], s["grad"], s["dX"],
               s["dW"], s["ws"])
    return s["loss"], s["lse"], s["dX"], s["dW"]


def run(state):
    return _own(state) if own else _plain(state)


# --------------------------------------------------------------------------------------- 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    op, n = case["op"], case["n"]

    def factor(n):
        """float64 [n]: 0 where element i is dropped, 1 / (1 - p') where it is kept (64-bit words)."""
        p, seed, call = case["p"], s["seed"], s["call"]
        thr = _threshold(p)
        if thr == 0:
            return torch.ones(n, device="cuda", dtype=torch.float64)
        u = np.uint64
        low, sh = u(_LOW), u(32)
        blk = np.arange((n + 7) // 8, dtype=np.uint64)
        c = [blk & low, blk >> sh, np.full_like(blk, call & _LOW),
             np.full_like(blk, (call >> 32) & _LOW)]
        key = [seed & _LOW, (seed >> 32) & _LOW]
        for _ in range(7):
            a, b = c[0] * u(_M0), c[2] * u(_M1)
            c = [(b >> sh) ^ c[1] ^ u(key[0]), b & low, (a >> sh) ^ c[3] ^ u(key[1]), a & low]
            key = [(key[0] + _K0) & _LOW, (key[1] + _K1) & _LOW]
        bits = np.stack(c, 1).astype("<u4").view("<u2").reshape(-1)[:n]
        kept = 1.0 / (1.0 - thr / 65536.0) if thr < 65536 else 0.0
        return torch.from_numpy(np.where(bits >= thr, kept, 0.0)).cuda()

    if op == "dropout_fwd":
        y = s["x"].double() * factor(n)
        return y + s["res"].double() if case["residual"] else y
    if op == "dropout_bwd":
        return s["dy"].double() * factor(n)
    H, V = case["H"], case["V"]
    if op == "embed_fwd":
        none = torch.zeros(1, H, device="cuda", dtype=torch.float64)
        padded = torch.cat([s["table"].double(), none])
        ids = torch.where(s["ids"] < 0, V, s["ids"].long())
        return padded[ids] * s["scale"] * factor(n * H).view(n, H)
    if op == "embed_bwd":
        g = s["dout"].double() * factor(n * H).view(n, H) * s["scale"]
        d = torch.zeros(V + 1, H, device="cuda", dtype=torch.float64)
        d.index_add_(0, torch.where(s["ids"] < 0, V, s["ids"].long()), g)
        return d[:V]
    # the labelled rows alone, a piece of them at a time
    rows = torch.nonzero(s["target"] >= 0)[:, 0]
    W = s["W"].double()
    loss = torch.zeros(n, device="cuda", dtype=torch.float64)
    lse = torch.zeros_like(loss)
    dX = torch.zeros(n, H, device="cuda", dtype=torch.float64)
    dW = torch.zeros(V, H, device="cuda", dtype=torch.float64)
    for at in rows.split(max(1, (1 << 28) // V)):
        x, t = s["X"][at].double(), s["target"][at].long()
        z = x @ W.t()
        lse[at] = torch.logsumexp(z, 1)
        loss[at] = lse[at] - z[torch.arange(len(at), device="cuda"), t]
        if op == "xent_train":
            d = torch.softmax(z, 1)
            d[torch.arange(len(at), device="cuda"), t] -= 1.0
            d *= s["dloss"][at].double()[:, None]
            dX[at] = d @ W
            dW += d.t() @ x
    return (loss, lse, dX, dW) if op == "xent_train" else (loss, lse)


# --------------------------------------------------------------------------------------- work


def _distinct(n, V):
    """Expected number of different ids among n drawn by _zipf."""
    w = 1.0 / np.arange(2, V + 2)
    return float(np.sum(-np.expm1(n * np.log1p(-w / w.sum()))))


def work(case):
    op, n = case["op"], case["n"]
    e = 4 if case.get("dtype", "f32") == "f32" else 2
    if op == "dropout_fwd":
        return {"bytes": n * e * (3 if case["residual"] else 2), "flops": 2 * n}
    if op == "dropout_bwd":
        return {"bytes": n * 8, "flops": n}
    H, V = case["H"], case["V"]
    if op == "embed_fwd":
        return {"bytes": n * 4 + _distinct(n - n // 50, V) * H * e + n * H * e, "flops": 2 * n * H}
    if op == "embed_bwd":
        return {"bytes": n * 4 + (n - n // 50) * H * 4 + V * H * 4, "flops": 2 * n * H}
    m = _labelled(case)
    moved = n * 4 + m * H * e + V * H * e + n * 8
    if op == "xent_fwd":
        return {"bytes": moved, "flops": 2 * m * V * H}
    g = 4 if case["grad"] == "f32" else 2
    # the logits, and the two products of the gradient
    return {"bytes": moved + m * 4 + n * H * g + V * H * g, "flops": 6 * m * V * H}
