"""Cases of the operators that answer with a vocabulary and learn from such answers: logits of states,
their adjustment (biases, penalties for repeated tokens, grammar masks), the top of a row of logits, and
distillation from a teacher's top logits, forward and with its gradient.

`listed()` / `draw()` give cases, `prepare()` a case's inputs, `run()` one pass (the library's calls
where `own` is true, elementary torch operations in 32 bits where it is not), `exact()` the same
outputs in 64 bits and `work()` the bytes and operations a pass cannot do without.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# --------------------------------------------------------------------------------------- cases


def listed():
    return [
        # one node's logits over the whole vocabulary: a completion request
        dict(name="logits_1", op="logits", n=1, H=128, V=32000, dtype="bf16", out="f32", pad=0),
        # one 20k-node graph in 32 bits
        dict(name="logits_f32_20k", op="logits", n=20001, H=128, V=32000, dtype="f32", out="f32", pad=0),
        # a teacher's logits for a sixth of a packed batch, widest state, largest vocabulary (odd rows)
        dict(name="logits_16k", op="logits", n=16383, H=256, V=49999, dtype="bf16", out="f32", pad=0),
        # the next tokens of eight completions at once: a short history and a grammar state each
        dict(name="adjust_8", op="adjust", n=8, V=32000, dtype="f32", pad=0, bias=True, masks=8, history=512),
        # the constraints of a large batch written into its logits, rows of an odd length
        dict(name="adjust_8k", op="adjust", n=8192, V=49999, dtype="bf16", pad=0, bias=True, masks=64,
             history=1024),
        # the suggestions of one completion request
        dict(name="top_1", op="top", n=1, V=32000, K=5, dtype="f32", pad=0, bias=False, masks=1, history=64),
        # a teacher's answer for one 2k-node graph: many entries, no constraints
        dict(name="top_f32_2k", op="top", n=2003, V=49999, K=64, dtype="f32", pad=1, bias=False, masks=0,
             history=0),
        # the teacher's answers for a large batch under a grammar, with biases and penalties
        dict(name="top_16k", op="top", n=16383, V=49999, K=32, dtype="bf16", pad=1, bias=True, masks=64,
             history=512),
        # validation of a student on the correctness workload's graph, in 32 bits
        dict(name="distill_eval_512", op="distill_fwd", n=512, H=64, V=4001, K=8, dtype="f32", tau=1.0,
             labelled=1.0),
        # validation on one 20k-node graph
        dict(name="distill_eval_20k", op="distill_fwd", n=20001, H=128, V=32000, K=32, dtype="bf16", tau=2.0,
             labelled=1.0),
        # a training step on a packed batch of which 15% of the nodes carry a teacher's answer
        dict(name="distill_train_masked_72k", op="distill_train", n=71969, H=64, V=10000, K=16, dtype="bf16",
             grad="f32", tau=2.0, labelled=0.15),
        # every node of half the largest supergraph, widest state, largest vocabulary
        dict(name="distill_train_65k", op="distill_train", n=65537, H=256, V=49999, K=32, dtype="bf16",
             grad="bf16", tau=2.0, labelled=1.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logits", "adjust", "top", "top", "distill_fwd", "distill_train", "distill_train"])
    V, dtype = _log_int(rng, 129, 49999), rng.choice(["f32", "bf16"])
    if op in ("adjust", "top"):
        case = dict(op=op, n=_log_int(rng, 1, 8192 if op == "adjust" else 16383), V=V, dtype=dtype,
                    pad=rng.choice([0, 0, 1, 3, 17]), bias=rng.random() < 0.5,
                    masks=rng.choice([0, 1, 7, 64]), history=rng.choice([0, 64, 512, 1024]))
        if op == "top":
            case["K"] = _log_int(rng, 1, 128)
        return case
    H = 32 * rng.randint(1, 8)
    if op == "logits":
        case = dict(op=op, n=_log_int(rng, 1, 20001), H=H, V=V, dtype=dtype,
                    out=rng.choice(["f32", "bf16"]), pad=rng.choice([0, 0, 1, 17]))
        most = 16383 * 49999 * 256 // (4 if dtype == "f32" else 1)
    else:
        case = dict(op=op, n=_log_int(rng, 1, 65537), H=H, V=V, K=_log_int(rng, 1, 128), dtype=dtype,
                    tau=rng.choice([1.0, 2.0, 3.5]), labelled=rng.choice([0.15, 0.5, 1.0]))
        if op == "distill_train":
            case["grad"] = "f32" if dtype == "f32" else rng.choice(["f32", "bf16"])
        most = 65537 * 49999 * 256 // (4 if dtype == "f32" else 1)
    # 32-bit inputs stay within a quarter of the largest case's products
    while case["n"] * V * H > most:
        case["n"] = (case["n"] + 1) // 2
    return case


# --------------------------------------------------------------------------------------- inputs


def _zipf(n, V, gen):
    """n ids in [0, V), id r drawn with weight 1 / (r + 2): token frequencies, in falling order."""
    w = 1.0 / torch.arange(2, V + 2, device="cuda", dtype=torch.float64)
    cdf = torch.cumsum(w, 0)
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) * cdf[-1]
    return torch.searchsorted(cdf, u).clamp_(max=V - 1).to(torch.int32)


def _rows(n, V, pad, dtype):
    """A [n, V] tensor whose rows are V + pad elements apart."""
    return torch.empty(n, V + pad, device="cuda", dtype=DTYPES[dtype])[:, :V]


def _constraints(s, gen):
    """The adjustment of a batch's logits: what a completion service holds for its requests."""
    n, V = s["n"], s["V"]
    # -100 bans a token, positive values favour those in scope
    s["bias_v"] = None
    if s["bias"]:
        b = torch.randn(V, generator=gen, device="cuda")
        s["bias_v"] = torch.where(torch.rand(V, generator=gen, device="cuda") < 0.01, -100.0, b)
    s["mask"] = s["mask_row"] = None
    if s["masks"]:
        # a state of the grammar allows between a hundredth and all of the tokens; with many states, the
        # first is a dead end, and some rows are under none (-1)
        G, words = s["masks"], (V + 31) // 32
        share = 10.0 ** (-2.0 * torch.rand(G, 1, generator=gen, device="cuda"))
        allowed = torch.rand(G, words * 32, generator=gen, device="cuda") < share
        low = 0
        if G > 8:
            allowed[0] = False
            low = -1
        bits = torch.arange(32, device="cuda")
        word = (allowed.view(G, words, 32).long() << bits).sum(2)
        s["mask"] = torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)
        s["mask_row"] = torch.randint(low, G, (n,), generator=gen, device="cuda", dtype=torch.int32)
    s["hist"] = s["hist_off"] = s["penalty"] = None
    if s["history"]:
        # histories of 0 to `history` tokens; repetition, presence and frequency penalties of each request
        size = torch.randint(0, s["history"] + 1, (n,), generator=gen, device="cuda")
        if n == 1:
            size[:] = s["history"]
        s["hist_off"] = torch.cat([size.new_zeros(1), size.cumsum(0)])
        s["hist"] = _zipf(int(size.sum()), V, gen)
        r = torch.rand(n, 3, generator=gen, device="cuda")
        s["penalty"] = torch.stack([1.0 + 0.5 * r[:, 0], r[:, 1], 0.5 * r[:, 2]], 1).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    s = dict(case)
    op, n, V = case["op"], case["n"], case["V"]
    if op in ("adjust", "top"):
        # logits of a trained model: the tokens' frequencies and what the state adds
        Z = _rows(n, V, case["pad"], case["dtype"])
        prior = torch.log(torch.arange(2, V + 2, device="cuda", dtype=torch.float32))
        for at in range(0, n, 2048):
            rows = Z[at:at + 2048]
            rows.copy_(2.5 * normal(*rows.shape) - 0.5 * prior)
        s["Z"] = Z
        _constraints(s, gen)
        return s
    H = case["H"]
    target = _zipf(n, V, gen)
    W = normal(V, H) * (2.0 / math.sqrt(H))
    # states that have learnt something about their tokens
    lean = 2.0 * torch.rand(n, 1, generator=gen, device="cuda")
    X = normal(n, H) + lean * W[target.long()]
    if op != "logits":
        # the teacher's top logits (rows it was not asked for have none, some rows fewer than K), and a
        # student that is on its way to them
        K = min(case["K"], V)
        s["K"] = K
        ids = torch.empty(n, K, device="cuda", dtype=torch.int32)
        top = torch.empty(n, K, device="cuda")
        Wt = W.to(torch.bfloat16)
        for at in range(0, n, 8192):
            z = X[at:at + 8192].to(torch.bfloat16) @ Wt.t()
            u, t = z.float().topk(K, 1)
            top[at:at + 8192], ids[at:at + 8192] = u, t.to(torch.int32)
        short = torch.rand(n, generator=gen, device="cuda") < 0.1
        ids[short, (K + 1) // 2:] = -1
        top[short, (K + 1) // 2:] = -math.inf
        m = max(1, int(round(case["labelled"] * n)))
        out = torch.rand(n, generator=gen, device="cuda").argsort()[m:]
        ids[out], top[out] = -1, -math.inf
        s["top_id"], s["top_logit"] = ids, top
        X = X + 0.5 * normal(n, H)
        W = W + normal(V, H) * (1.0 / math.sqrt(H))
        if op == "distill_train":
            # the mean over the rows that count, each with a weight of its own
            s["dloss"] = (0.5 + torch.rand(n, generator=gen, device="cuda")) / m
    s["X"], s["W"] = X.to(DTYPES[case["dtype"]]), W.to(DTYPES[case["dtype"]])
    return s


# --------------------------------------------------------------------------------------- plain form


def _allowed(s):
    """bool [masks, V]: bit v % 32 of word v / 32."""
    v = torch.arange(s["V"], device="cuda")
    return ((s["mask"][:, v // 32] >> (v % 32).to(torch.int32)) & 1) != 0


def _counts(s):
    """float [n, V]: how often each token is in each row's history."""
    n, V, off = s["n"], s["V"], s["hist_off"]
    row = torch.repeat_interleave(torch.arange(n, device="cuda"), off[1:] - off[:-1],
                                  output_size=s["hist"].numel())
    c = torch.zeros(n * V, device="cuda")
    c.scatter_add_(0, row * V + s["hist"], torch.ones(row.numel(), device="cuda"))
    return c.view(n, V)


def _adjusted(s):
    """The adjusted logits in 32 bits, every operation rounded: the bias, then the penalties, then the mask."""
    z = s["Z"].float()
    if s["bias_v"] is not None:
        z = z + s["bias_v"]
    if s["penalty"] is not None:
        c = _counts(s)
        rep, presence, frequency = s["penalty"][:, 0:1], s["penalty"][:, 1:2], s["penalty"][:, 2:3]
        less = torch.where(z > 0, z / rep, z * rep) - (presence + frequency * c)
        z = torch.where(c > 0, less, z)
    if s["mask"] is not None:
        row = s["mask_row"].long()
        keep = _allowed(s)[row.clamp(min=0)] | (row < 0)[:, None]
        z = torch.where(keep, z, torch.full_like(z, -math.inf))
    return z


def _top(s):
    z = _adjusted(s)
    n, V, K = s["n"], s["V"], min(s["K"], s["V"])
    # keys of 64 bits: the value's order, then the lower id
    bits = (z + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    key = order * 2 ** 31 + (V - 1 - torch.arange(V, device="cuda"))
    best = key.topk(K, 1).values
    ids = V - 1 - (best & (2 ** 31 - 1))
    top = z.gather(1, ids)
    ids = torch.where(top > -math.inf, ids, torch.full_like(ids, -1)).to(torch.int32)
    high = top[:, :1].clamp(min=-3.0e38)
    lse = (high + torch.log(torch.exp(z - high).sum(1, keepdim=True)))[:, 0]
    return top, ids, lse


def _distill(s):
    X, W, tau = s["X"].float(), s["W"].float(), s["tau"]
    ids = s["top_id"].long()
    there = ids >= 0
    valid = there.any(1)
    X = torch.where(valid[:, None], X, torch.zeros_like(X))
    z = X @ W.t() / tau
    u = torch.where(there, s["top_logit"] / tau, torch.full_like(s["top_logit"], -math.inf))
    high = torch.where(valid, u.amax(1), torch.zeros_like(u[:, 0]))[:, None]
    e = torch.exp(u - high)
    total = e.sum(1, keepdim=True).clamp(min=1e-30)
    q = e / total
    log_q = torch.where(there, u - high - torch.log(total), torch.zeros_like(u))
    top = z.amax(1, keepdim=True)
    probs = torch.exp(z - top)
    part = probs.sum(1, keepdim=True)
    lse = torch.where(valid, (top + torch.log(part))[:, 0], torch.zeros_like(top[:, 0]))
    at = ids.clamp(min=0)
    inner = torch.where(there, q * (log_q - z.gather(1, at)), torch.zeros_like(u)).sum(1)
    loss = torch.where(valid, tau * tau * (inner + lse), torch.zeros_like(lse))
    if s["op"] == "distill_fwd":
        return loss, lse
    probs *= 1.0 / part
    probs.scatter_add_(1, at, -q)
    probs *= torch.where(valid, s["dloss"] * tau, torch.zeros_like(lse))[:, None]
    out = DTYPES[s["grad"]]
    return loss, lse, (probs @ W).to(out), (probs.t() @ X).to(out)


def _plain(s):
    if s["op"] == "logits":
        return (s["X"].float() @ s["W"].float().t()).to(DTYPES[s["out"]])
    if s["op"] == "adjust":
        return _adjusted(s).to(DTYPES[s["dtype"]])
    if s["op"] == "top":
        return _top(s)
    return _distill(s)


# ------------------------------------------------------------------------------ the library


def _own(s):
    from paper_1906_11786_gb300 import lib as L

    op, n, V, dtype = s["op"], s["n"], s["V"], s["dtype"]

    def scratch(size):
        return torch.empty(max(size, 256), device="cuda", dtype=torch.uint8)

    if op == "logits":
        if "out_z" not in s:
            s["out_z"] = _rows(n, V, s["pad"], s["out"])
            s["ws"] = scratch(L.logits_workspace_bytes(dtype, n, s["H"], V))
        L.logits_fwd(dtype, s["X"], s["W"], s["out"], s["out_z"], s["ws"])
        return s["out_z"]
    if op in ("adjust", "top"):
        if "adjust" not in s:
            s["adjust"] = L.LogitAdjust(bias=s["bias_v"], mask=s["mask"], mask_row=s["mask_row"],
                                        history=s["hist"], history_off=s["hist_off"],
                                        penalty=s["penalty"])
        if op == "adjust":
            if "out_z" not in s:
                s["out_z"] = _rows(n, V, s["pad"], dtype)
            L.logits_adjust(dtype, s["Z"], s["out_z"], s["adjust"])
            return s["out_z"]
        if "top" not in s:
            K = min(s["K"], V)
            s["top"] = torch.empty(n, K, device="cuda")
            s["ids"] = torch.empty(n, K, device="cuda", dtype=torch.int32)
            s["lse"] = torch.empty(n, device="cuda")
        L.logits_top(dtype, s["Z"], s["top"], s["ids"], s["lse"], s["adjust"])
        return s["top"], s["ids"], s["lse"]
    H, K, tau = s["H"], s["K"], s["tau"]
    if "loss" not in s:
        s["loss"], s["lse"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        need = L.distill_workspace_bytes(dtype, n, H, V, K, L.BG_OP_DISTILL_FWD)
        if op == "distill_train":
            s["dX"] = torch.empty(n, H, device="cuda", dtype=DTYPES[s["grad"]])
            s["dW"] = torch.empty(V, H, device="cuda", dtype=DTYPES[s["grad"]])
            need = max(need, L.distill_workspace_bytes(dtype, n, H, V, K, L.BG_OP_DISTILL_BWD))
        s["ws"] = scratch(need)
    L.distill_fwd(dtype, s["X"], s["W"], s["top_id"], s["top_logit"], s["loss"], s["lse"], s["ws"],
                  tau=tau)
    if op == "distill_fwd":
        return s["loss"], s["lse"]
    L.distill_bwd(dtype, s["X"], s["W"], s["top_id"], s["top_logit"], s["lse"], s["dloss"], s["grad"],
                  s["dX"], s["dW"], s["ws"], tau=tau)
    return s["loss"], s["lse"], s["dX"], s["dW"]


def run(state):
    return _own(state) if own else _plain(state)


# --------------------------------------------------------------------------------------- 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    op, n, V = case["op"], case["n"], case["V"]
    f64 = torch.float64
    if op == "logits":
        Z = torch.empty(n, V, device="cuda", dtype=f64)
        W = s["W"].double()
        for at in range(0, n, 4096):
            Z[at:at + 4096] = s["X"][at:at + 4096].double() @ W.t()
        return Z
    if op in ("adjust", "top"):
        out, tops, lses = [], [], []
        grid = torch.arange(V, device="cuda")
        for at in range(0, n, 2048):
            z = s["Z"][at:at + 2048].double()
            rows = z.shape[0]
            if s["bias_v"] is not None:
                z += s["bias_v"].double()
            if s["penalty"] is not None:
                off = s["hist_off"][at:at + rows + 1]
                ids = s["hist"][int(off[0]):int(off[-1])].long()
                line = torch.searchsorted(off, torch.arange(int(off[0]), int(off[-1]), device="cuda"),
                                          right=True) - 1
                cell, count = torch.unique(line * V + ids, return_counts=True)
                r, c = cell // V, cell % V
                p = s["penalty"][at:at + rows].double()[r]
                v = z[r, c]
                z[r, c] = v * p[:, 0] ** -torch.sign(v) - p[:, 1] - p[:, 2] * count
            if s["mask"] is not None:
                for g in range(s["masks"]):
                    ok = torch.bitwise_right_shift(s["mask"][g].long()[grid // 32], grid % 32) % 2 == 1
                    under = s["mask_row"][at:at + rows] == g
                    z.masked_fill_(under[:, None] & ~ok[None, :], -math.inf)
            if op == "adjust":
                out.append(z)
            else:
                tops.append(torch.sort(z, 1, descending=True).values[:, :case["K"]].clone())
                lses.append(torch.logsumexp(z, 1))
        return torch.cat(out) if op == "adjust" else (torch.cat(tops), None, torch.cat(lses))
    H, tau, K = case["H"], case["tau"], s["K"]
    loss = torch.zeros(n, device="cuda", dtype=f64)
    lse = torch.zeros_like(loss)
    dX, dW = torch.zeros(n, H, device="cuda", dtype=f64), torch.zeros(V, H, device="cuda", dtype=f64)
    W = s["W"].double()
    # the rows with a teacher's answer alone, a piece of them at a time
    for at in torch.nonzero(s["top_id"][:, 0] >= 0)[:, 0].split(max(1, (1 << 28) // V)):
        x, t = s["X"][at].double(), s["top_id"][at].long()
        logp = torch.log_softmax(x @ W.t() / tau, 1)
        u = s["top_logit"][at].double() / tau
        q = torch.softmax(u, 1)
        some = t >= 0
        pick = logp.gather(1, t * some)
        loss[at] = tau ** 2 * torch.where(some, torch.xlogy(q, q) - q * pick, 0.0).sum(1)
        lse[at] = (x * W[t[:, 0]]).sum(1) / tau - pick[:, 0]
        if op == "distill_train":
            d = logp.exp_()
            d.scatter_add_(1, t * some, -q)
            d *= (tau * s["dloss"][at].double())[:, None]
            dX[at] = d @ W
            dW += d.t() @ x
    return (loss, lse, dX, dW) if op == "distill_train" else (loss, lse)


# --------------------------------------------------------------------------------------- work


def work(case):
    op, n, V = case["op"], case["n"], case["V"]
    e = 4 if case["dtype"] == "f32" else 2
    if op == "logits":
        H = case["H"]
        return {"bytes": (n + V) * H * e + n * V * (4 if case["out"] == "f32" else 2),
                "flops": 2 * n * V * H}
    if op in ("adjust", "top"):
        # histories are half of the longest on average
        side = (V * 4 if case["bias"] else 0) + case["masks"] * V // 8 + n * case["history"] * 2
        out = n * V * e if op == "adjust" else n * (case["K"] * 8 + 4)
        return {"bytes": n * V * e + side + out, "flops": n * V * (2 if op == "adjust" else 4)}
    H, K = case["H"], min(case["K"], V)
    m = max(1, int(round(case["labelled"] * n)))
    moved = m * H * e + V * H * e + n * K * 8 + n * 8
    if op == "distill_fwd":
        return {"bytes": moved, "flops": 2 * m * V * H}
    g = 4 if case["grad"] == "f32" else 2
    # the logits, and the two products of the gradient
    return {"bytes": moved + m * 4 + n * H * g + V * H * g, "flops": 6 * m * V * H}
