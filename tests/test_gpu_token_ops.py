"""GPU parity of the token operators (dropout, embedding, vocabulary cross entropy) against plain
64-bit implementations, at the sizes, masks and values where they can go wrong.

Every bound below is derived from the arithmetic the operators promise; u = 2^-24 is half the gap of
fp32, and a result rounded to bf16 adds 2^-8 of itself.
"""
from __future__ import annotations

import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import token_ref as ref
from gpu_common import ensure_built
from paper_1906_11786_gb300 import _binding as L

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = 2.0 ** -8  # rounding to bf16 (8 significant bits), relative
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
SEED, CALL = 0x1906_1178_6000_0001, 0x7FFF_0000_1234


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()


def dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(TD[dtype]).cuda()


def host(t):
    return t.double().cpu().numpy()


def within(got, want, tol, what=""):
    """|got - want| <= tol element by element (tol an array or a number)."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape
    over = np.abs(got - want) - tol
    assert np.all(np.isfinite(got)), f"{what}: not finite"
    assert over.size == 0 or over.max() <= 0, \
        f"{what}: {np.abs(got - want).flat[over.argmax()]:.3e} off at {over.argmax()}"


# ------------------------------------------------------------------------------ dropout


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 2048, 4097, 100003])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(dtype, n, p):
    rng = np.random.default_rng(n)
    x, r = dev(rng.standard_normal(n), dtype), dev(rng.standard_normal(n), dtype)
    for res in (None, r):
        y = torch.full_like(x, float("nan"))
        L.dropout_fwd(dtype, x, y, p, SEED, CALL, residual=res)
        d = ref.drop(host(x), p, SEED, CALL)
        want = d + (host(r) if res is not None else 0.0)
        # the scale, its product and the sum: one rounding each
        tol = 2 * U * np.abs(d) + U * np.abs(want) * 1.01
        within(host(y), want, tol + (HALF * 1.01 * np.abs(want) if dtype == "bf16" else 0))
    if dtype == "f32":
        dx = x.clone()
        L.dropout_bwd(r, dx, p, SEED, CALL, flags=L.BG_ACCUM)
        d = ref.drop(host(r), p, SEED, CALL)
        within(host(dx), host(x) + d, 2 * U * np.abs(d) + U * 1.01 * np.abs(host(x) + d))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [2490367, 5000011, 23000005])
def test_dropout_of_millions_of_elements(dtype, n):
    """Every element of sizes at which a thread has one group of 8, several, and results that are not kept
    in the cache (past 128 MB of operands), each with a rest."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    x, r = (torch.randn(n, device="cuda", generator=gen).to(TD[dtype]) for _ in range(2))
    p = 0.3
    d = ref.drop(host(x), p, SEED, CALL)
    for res in (None, r):
        y = torch.full_like(x, float("nan"))
        L.dropout_fwd(dtype, x, y, p, SEED, CALL, residual=res)
        want = d + (host(r) if res is not None else 0.0)
        tol = 2 * U * np.abs(d) + U * np.abs(want) * 1.01
        within(host(y), want, tol + (HALF * 1.01 * np.abs(want) if dtype == "bf16" else 0))
    if dtype == "f32":
        for flags, before in ((0, 0.0), (L.BG_ACCUM, host(r))):
            dx = r.clone()
            L.dropout_bwd(x, dx, p, SEED, CALL, flags=flags)
            within(host(dx), before + d, 2 * U * np.abs(d) + U * 1.01 * np.abs(before + d))


def test_dropout_of_half_the_bytes_takes_no_longer():
    """bf16 elements are read and written 16 bytes at a time too, at sizes where a thread has one group of 8:
    element by element they took 1.7 times as long as fp32 ones (now 0.8)."""
    n = 2490368
    times = {}
    for dtype in ("f32", "bf16"):
        x = torch.ones(n, device="cuda", dtype=TD[dtype])
        y = torch.empty_like(x)
        L.dropout_fwd(dtype, x, y, 0.1, SEED, CALL)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(50):
                L.dropout_fwd(dtype, x, y, 0.1, SEED, CALL)
        best = []
        for _ in range(8):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            graph.replay()
            b.record()
            b.synchronize()
            best.append(a.elapsed_time(b))
        times[dtype] = min(best)
    assert times["bf16"] < 1.2 * times["f32"], times


def test_dropout_keeps_the_stated_share():
    """Kept elements are binomial: within 6 standard deviations of (1 - p) n for every p, and masks of
    different calls agree as often as independent ones do."""
    n = 1 << 20
    x, y = torch.ones(n, device="cuda"), torch.empty(n, device="cuda")
    for p in (0.1, 0.25, 0.5, 0.9):
        L.dropout_fwd("f32", x, y, p, SEED, CALL)
        share = 1 - round(p * 65536) / 65536
        assert abs(int((y != 0).sum()) - share * n) < 6 * np.sqrt(n * share * (1 - share))
    L.dropout_fwd("f32", x, y, 0.5, SEED, CALL)
    z = torch.empty_like(y)
    for seed, call in ((SEED + 1, CALL), (SEED, CALL + 1)):
        L.dropout_fwd("f32", x, z, 0.5, seed, call)
        assert abs(int(((y != 0) == (z != 0)).sum()) - n / 2) < 6 * np.sqrt(n / 4)


def test_dropout_in_place_and_with_values_that_are_not_finite():
    n, p = 1003, 0.5
    k = ref.keep(0, n, p, SEED, CALL)
    x = torch.where(torch.from_numpy(k).cuda(), torch.ones(n, device="cuda"),
                    torch.full((n,), float("nan"), device="cuda"))
    r = torch.arange(n, device="cuda", dtype=torch.float32)
    y = r.clone()
    L.dropout_fwd("f32", x, y, p, SEED, CALL, residual=y)  # y is the residual
    assert torch.equal(y, r + 2.0 * torch.from_numpy(k).cuda())
    L.dropout_fwd("f32", x, x, p, SEED, CALL)  # y is x
    assert torch.equal(x, 2.0 * torch.from_numpy(k).cuda().float())
    bad = torch.tensor([float("inf"), float("nan")] * 500, device="cuda")
    out = torch.empty_like(bad)
    L.dropout_fwd("f32", bad, out, 1.0, SEED, CALL)
    assert torch.count_nonzero(out) == 0


def test_dropout_past_32_bits_of_elements():
    n = (1 << 32) + 11
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    L.dropout_fwd("bf16", x, x, 0.25, SEED, CALL)
    for first in (0, (1 << 31) - 5, (1 << 32) - 5, n - 16):
        got = (x[first:first + 16] != 0).cpu().numpy()
        assert np.array_equal(got, ref.keep(first, len(got), 0.25, SEED, CALL))


# ------------------------------------------------------------------------------ embedding


def make_ids(rng, n, V, kind):
    if kind == "uniform":
        return rng.integers(0, V, n).astype(np.int32)
    if kind == "one":  # every row the same token
        return np.full(n, V // 2, np.int32)
    if kind == "none":
        return np.full(n, -1, np.int32)
    w = 1.0 / np.arange(2, V + 2)  # frequent and rare tokens, every fifth row padding
    ids = rng.choice(V, n, p=w / w.sum()).astype(np.int32)
    ids[rng.random(n) < 0.2] = -1
    return ids


EMBED = [(1, 32, 1, "uniform"), (2, 64, 2, "uniform"), (31, 96, 3, "zipf"), (33, 256, 40, "one"),
         (512, 64, 1000, "zipf"), (2047, 160, 511, "zipf"), (2049, 128, 512, "uniform"),
         (5000, 224, 513, "zipf"), (4100, 64, 70000, "uniform"), (9000, 32, 300000, "zipf"),
         (70001, 32, 17, "zipf"), (20000, 256, 30, "one"), (100, 64, 50, "none")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,H,V,kind", EMBED)
def test_embed_fwd(dtype, n, H, V, kind):
    rng = np.random.default_rng(n + H)
    ids = make_ids(rng, n, V, kind)
    table, scale = dev(rng.standard_normal((V, H)), dtype), 1.7
    for p in (0.0, 0.3):
        out = torch.full((n, H), float("nan"), device="cuda", dtype=TD[dtype])
        L.embed_fwd(dtype, torch.from_numpy(ids).cuda(), table, out, scale=scale, p=p, seed=SEED,
                    call=CALL)
        want = ref.embed_fwd(ids, host(table), float(np.float32(scale)), p, SEED, CALL)
        # scale * kept scale (rounded), two products
        tol = 3.01 * U * np.abs(want) + (1.01 * HALF * np.abs(want) if dtype == "bf16" else 0)
        within(host(out), want, tol)


@pytest.mark.parametrize("n,H,V,kind", EMBED)
def test_embed_bwd(n, H, V, kind):
    rng = np.random.default_rng(n + H)
    ids = make_ids(rng, n, V, kind)
    dout, scale = rng.standard_normal((n, H)).astype(np.float32), 0.6
    dout[ids < 0] = np.nan  # padding rows are not read
    d_ids, d_out = torch.from_numpy(ids).cuda(), torch.from_numpy(dout).cuda()
    ws = torch.empty(L.embed_workspace_bytes(n, H, V), device="cuda", dtype=torch.uint8)
    for p in (0.0, 0.3):
        want, mag, count = ref.embed_bwd(ids, np.nan_to_num(dout), V, float(np.float32(scale)), p,
                                         SEED, CALL)
        # a sum of `count` terms in fp32, its scale and the product
        tol = (count[:, None] + 3) * U * mag
        got = torch.full((V, H), float("nan"), device="cuda")
        ws.fill_(0xA5)
        L.embed_bwd(d_ids, d_out, got, ws, scale=scale, p=p, seed=SEED, call=CALL)
        within(host(got), want, tol)
        again = torch.full((V, H), float("nan"), device="cuda")
        ws.fill_(0x5A)
        L.embed_bwd(d_ids, d_out, again, ws, scale=scale, p=p, seed=SEED, call=CALL)
        assert torch.equal(got, again), "the sum's order is fixed"
        base = torch.from_numpy(rng.standard_normal((V, H)).astype(np.float32)).cuda()
        acc = base.clone()
        L.embed_bwd(d_ids, d_out, acc, ws, scale=scale, p=p, seed=SEED, call=CALL, flags=L.BG_ACCUM)
        assert torch.equal(acc, base + got), "BG_ACCUM adds the finished sum"


# (rows, H, V): the largest sort of one cluster; then counting passes of many blocks: two and three
# passes, one tile of keys a block and several, all keys of one digit
SORTS = [(32768, 32, 600, "uniform"), (32769, 32, 600, "uniform"), (40001, 64, 5000, "one"),
         (100003, 64, 49999, "zipf"), (50001, 32, 300000, "zipf"), (330000, 32, 1 << 18, "uniform"),
         (700001, 32, 5000, "zipf")]


@pytest.mark.parametrize("n,H,V,kind", SORTS)
def test_embed_bwd_of_many_ids(n, H, V, kind):
    """Integers as gradients: every sum is exact in fp32, so that a row in the wrong place, lost or taken
    twice shows, whatever the order of additions."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    ids = torch.from_numpy(make_ids(np.random.default_rng(n + V), n, V, kind)).cuda()
    dout = torch.randint(-9, 10, (n, H), generator=gen, device="cuda").float()
    dout[ids < 0] = float("nan")  # padding rows are not read
    want = torch.zeros(V, H, device="cuda", dtype=torch.float64)
    want.index_add_(0, ids[ids >= 0].long(), dout[ids >= 0].double())
    ws = torch.empty(L.embed_workspace_bytes(n, H, V), device="cuda", dtype=torch.uint8)
    for fill in (0xA5, 0x5A):
        got = torch.full((V, H), float("nan"), device="cuda")
        ws.fill_(fill)
        L.embed_bwd(ids, dout, got, ws, scale=2.0)
        assert torch.equal(got.double(), 2.0 * want)
    base = torch.randint(-9, 10, (V, H), generator=gen, device="cuda").float()
    acc = base.clone()
    L.embed_bwd(ids, dout, acc, ws, scale=2.0, flags=L.BG_ACCUM)
    assert torch.equal(acc.double(), base + 2.0 * want)
    # real values with dropout: the same bits again, and the sums of the formula
    real = torch.randn(n, H, generator=gen, device="cuda")
    outs = []
    for fill in (0xA5, 0x5A):
        outs.append(torch.full((V, H), float("nan"), device="cuda"))
        ws.fill_(fill)
        L.embed_bwd(ids, real, outs[-1], ws, scale=0.6, p=0.3, seed=SEED, call=CALL)
    assert torch.equal(*outs)
    kept = torch.from_numpy(ref.drop(np.ones((n, H)), 0.3, SEED, CALL)).cuda() * real.double()
    ok = ids >= 0
    want, mag = (torch.zeros(V, H, device="cuda", dtype=torch.float64).index_add_(
        0, ids[ok].long(), v[ok] * float(np.float32(0.6))) for v in (kept, kept.abs()))
    count = torch.bincount(ids[ok].long(), minlength=V).double()[:, None]
    within(host(outs[0]), host(want), host((count + 3) * U * mag))
    L.check_device()


def test_embed_gradient_is_the_adjoint():
    """<embed(D), G> = <D, embed_bwd(G)>: the lookup is linear in its table, so differences of it are
    the lookup itself.  Both sides are sums of n H products of fp32 values with a few roundings each."""
    n, H, V, p = 3001, 64, 257, 0.25
    rng = np.random.default_rng(5)
    ids = torch.from_numpy(make_ids(rng, n, V, "zipf")).cuda()
    D = torch.from_numpy(rng.standard_normal((V, H)).astype(np.float32)).cuda()
    G = torch.from_numpy(rng.standard_normal((n, H)).astype(np.float32)).cuda()
    out, dD = torch.empty(n, H, device="cuda"), torch.empty(V, H, device="cuda")
    ws = torch.empty(L.embed_workspace_bytes(n, H, V), device="cuda", dtype=torch.uint8)
    L.embed_fwd("f32", ids, D, out, scale=1.5, p=p, seed=SEED, call=CALL)
    L.embed_bwd(ids, G, dD, ws, scale=1.5, p=p, seed=SEED, call=CALL)
    a, b = float((out.double() * G).sum()), float((D.double() * dD).sum())
    mag = float((out.double() * G).abs().sum())
    assert abs(a - b) <= (n + 8) * U * mag


def test_embed_reports_ids_past_the_table():
    L.check_device()
    ids = torch.tensor([3, 9, 10, 2 ** 31 - 1, -7, 0], device="cuda", dtype=torch.int32)
    table = torch.arange(640, device="cuda", dtype=torch.float32).reshape(10, 64) + 1
    out = torch.full((6, 64), float("nan"), device="cuda")
    L.embed_fwd("f32", ids, table, out)
    with pytest.raises(L.BandGGNNError, match="site 130"):
        L.check_device()
    L.check_device()
    assert torch.equal(out[[0, 1, 5]], table[[3, 9, 0]]) and torch.count_nonzero(out[2:5]) == 0
    d = torch.full((10, 64), float("nan"), device="cuda")
    ws = torch.empty(L.embed_workspace_bytes(6, 64, 10), device="cuda", dtype=torch.uint8)
    L.embed_bwd(ids, torch.ones(6, 64, device="cuda"), d, ws)
    with pytest.raises(L.BandGGNNError, match="site 130"):
        L.check_device()
    want = torch.zeros(10, 64, device="cuda")
    want[[3, 9, 0]] = 1
    assert torch.equal(d, want)


def test_embed_of_no_rows():
    d = torch.full((7, 64), float("nan"), device="cuda")
    none = torch.empty(0, device="cuda", dtype=torch.int32)
    ws = torch.empty(L.embed_workspace_bytes(0, 64, 7), device="cuda", dtype=torch.uint8)
    L.embed_bwd(none, torch.empty(0, 64, device="cuda"), d, ws, flags=L.BG_ACCUM)
    assert torch.isnan(d).all()
    L.embed_bwd(none, torch.empty(0, 64, device="cuda"), d, ws)
    assert torch.count_nonzero(d) == 0


def test_embed_past_32_bits_of_elements():
    """n H just over 2^31: the last rows' offsets need 64 bits, forward and backward."""
    n, H, V = (1 << 23) + 5, 256, 3
    ids = torch.full((n,), -1, device="cuda", dtype=torch.int32)
    ids[-4:] = torch.tensor([0, 2, 1, 2], device="cuda", dtype=torch.int32)
    table = torch.arange(V * H, device="cuda", dtype=torch.float32).reshape(V, H)
    out = torch.empty(n, H, device="cuda")
    L.embed_fwd("f32", ids, table, out)
    assert torch.equal(out[-4:], table[[0, 2, 1, 2]]) and torch.count_nonzero(out[:-4]) == 0
    d = torch.empty(V, H, device="cuda")
    ws = torch.empty(L.embed_workspace_bytes(n, H, V), device="cuda", dtype=torch.uint8)
    L.embed_bwd(ids, out, d, ws)
    assert torch.equal(d, table * torch.tensor([1.0, 1.0, 2.0], device="cuda")[:, None])


# ------------------------------------------------------------------------------ cross entropy


def xent_inputs(n, H, V, dtype, share=1.0, zscale=2.0, seed=0):
    rng = np.random.default_rng(seed + n + H + V)
    W = rng.standard_normal((V, H)) * zscale / np.sqrt(H)
    target = rng.integers(0, V, n).astype(np.int32)
    X = rng.standard_normal((n, H)) + rng.random((n, 1)) * 2 * W[target]
    target[rng.random(n) >= share] = -1
    g = (0.5 + rng.random(n)).astype(np.float32) / max(n, 1)
    return dev(X, dtype), dev(W, dtype), target, g


def run_xent(dtype, X, W, target, g, grad, flags=0, into=None):
    n, (V, H) = target.size, W.shape
    t, gd = torch.from_numpy(target).cuda(), torch.from_numpy(g).cuda()
    loss, lse = (torch.full((n,), float("nan"), device="cuda") for _ in range(2))
    need = max(L.xent_workspace_bytes(dtype, n, H, V, op) for op in (L.BG_OP_XENT_FWD,
                                                                   L.BG_OP_XENT_BWD))
    ws = torch.full((need,), 0xA5, device="cuda", dtype=torch.uint8)
    L.xent_fwd(dtype, X, W, t, loss, lse, ws)
    dX, dW = into or (torch.full((m, H), float("nan"), device="cuda", dtype=TD[grad])
                      for m in (n, V))
    ws.fill_(0x5A)
    L.xent_bwd(dtype, X, W, t, lse, gd, grad, dX, dW, ws, flags=flags)
    return loss, lse, dX, dW


def xent_bounds(r, n, H, V, grad):
    """Element bounds.  A logit: H products to 21 bits or better, added in fp32 (at most H u of their
    magnitude, the tensor core's truncating adds included as 2 u each).  exp and log: 2^-20 of
    themselves, of arguments that carry the logits' error.  A gradient element: each term is off by
    the error of its probability and of its representation in the product (2^-19, and in bf16 twice
    2^-8: the probability's rounding and the result's), and the sums add V u or n u of the terms'
    magnitude.  A probability keeps its bits down to an absolute 2^-38 (for dW: of the largest weight),
    below which it may be lost, as everything below 2^-126 is."""
    dz = (2 * H * U + 2.0 ** -21) * r["zabs"]
    loss = 2 * dz + 2.0 ** -20 * (1 + np.abs(r["lse"]))
    term = 2 * dz + 2.0 ** -19 + (2.0 ** -7 if grad == "bf16" else 0)
    bX = (term + 2 * V * U) * r["absX"] + 2.0 ** -38 * r["allX"] + 2.0 ** -126
    bW = (term + 2 * n * U) * r["absW"] + 2.0 ** -38 * r["allW"] + 2.0 ** -126
    return loss, bX, bW


def rel2(got, want):
    """2-norm of the difference over that of the result."""
    return float(np.linalg.norm(host(got) - want) / max(np.linalg.norm(want), 1e-300))


def check_xent(dtype, grad, X, W, target, g, share_used=None):
    n, (V, H) = target.size, W.shape
    got = run_xent(dtype, X, W, target, g, grad)
    r = ref.xent(host(X), host(W), target, g)
    loss, bX, bW = xent_bounds(r, n, H, V, grad)
    used = (target >= 0) & (target < V)
    within(host(got[1]), r["lse"], loss * used, "lse")
    within(host(got[0]), r["loss"], loss * used, "loss")
    within(host(got[2]), r["dX"], bX, "dX")
    within(host(got[3]), r["dW"], bW, "dW")
    # over all elements roundings average out: 2^-16 of the norm in fp32, where it is not small by
    # cancellation, and 2^-8 in bf16
    if V > 1 and used.any():
        lim = 2.0 ** -8 if grad == "bf16" else 2.0 ** -16
        assert rel2(got[2], r["dX"]) < lim and rel2(got[3], r["dW"]) < lim
    return got


TYPES = [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")]
XENT = [(1, 32, 1, 1.0), (1, 64, 2, 1.0), (2, 128, 1000, 1.0), (1, 256, 4099, 1.0),
        (63, 96, 65, 1.0), (127, 64, 127, 0.5), (128, 160, 128, 1.0), (129, 192, 257, 0.7),
        (300, 224, 513, 0.15), (513, 256, 1023, 1.0), (1000, 32, 3001, 1.0), (2500, 64, 400, 0.15),
        (4097, 128, 130, 1.0), (700, 256, 2049, 0.02)]


@pytest.mark.parametrize("dtype,grad", TYPES)
@pytest.mark.parametrize("n,H,V,share", XENT)
def test_xent(dtype, grad, n, H, V, share):
    check_xent(dtype, grad, *xent_inputs(n, H, V, dtype, share))


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_xent_of_larger_shapes(dtype, grad):
    """Several tiles a block in both directions, every row of each side checked."""
    check_xent(dtype, grad, *xent_inputs(9001, 64, 6007, dtype, 0.9))
    check_xent(dtype, grad, *xent_inputs(3001, 256, 9001, dtype, 0.9))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 70, 130, 256, 257, 700, 1024])
def test_xent_of_many_rows_against_few_tokens(dtype, V):
    """Several tiles of rows a block, each of one to four pieces of the vocabulary: the four quarters of a
    tile's columns are joined within the block, whose warps do not wait for one another otherwise.  Every
    row, twenty times over."""
    n, H = 150001, 32
    X, W, target, g = xent_inputs(n, H, V, dtype, 0.9)
    t = torch.from_numpy(target).cuda()
    ws = torch.empty(L.xent_workspace_bytes(dtype, n, H, V, L.BG_OP_XENT_FWD), device="cuda",
                     dtype=torch.uint8)
    z = X.double() @ W.double().T
    ok = t >= 0
    want_lse = torch.where(ok, torch.logsumexp(z, 1), 0.0)
    want = torch.where(ok, want_lse - z.gather(1, t.clamp(min=0).long()[:, None])[:, 0], 0.0)
    zabs = float((X.double().abs() @ W.double().abs().T).max())
    tol = 2 * (2 * H * U + 2.0 ** -21) * zabs + 2.0 ** -20 * (1 + want_lse.abs())
    for _ in range(20):
        loss, lse = (torch.full((n,), float("nan"), device="cuda") for _ in range(2))
        L.xent_fwd(dtype, X, W, t, loss, lse, ws)
        for got, right in ((lse, want_lse), (loss, want)):
            over = (got.double() - right).abs() - tol
            assert float(over.max()) <= 0, (int(over.argmax()), float(over.max()))
    L.check_device()


@pytest.mark.parametrize("dtype,grad", TYPES)
@pytest.mark.parametrize("n,H,V,share", [(40001, 96, 300, 0.9), (70001, 32, 130, 0.9),
                                         (600001, 32, 40, 0.5)])
def test_xent_of_many_rows(dtype, grad, n, H, V, share):
    """Rows that are counted before they are gathered, in blocks of 64, of 256 and of two times 256."""
    check_xent(dtype, grad, *xent_inputs(n, H, V, dtype, share))


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_xent_of_confident_and_of_wrong_rows(dtype, grad):
    """Logits in the hundreds: softmax is all but one-hot, right or wrong, and nothing overflows."""
    X, W, target, g = xent_inputs(260, 64, 301, dtype, 1.0, zscale=40.0)
    check = host(X) @ host(W).T
    assert np.abs(check).max() > 300
    got = run_xent(dtype, X, W, target, g, grad)
    r = ref.xent(host(X), host(W), target, g)
    loss, bX, bW = xent_bounds(r, 260, 64, 301, grad)
    for t, w, b in zip(got, (r["loss"], r["lse"], r["dX"], r["dW"]), (loss, loss, bX, bW)):
        within(host(t), w, b)


def check_bounds(dtype, grad, X, W, target, g):
    n, (V, H) = target.size, W.shape
    got = run_xent(dtype, X, W, target, g, grad)
    r = ref.xent(host(X), host(W), target, g)
    loss, bX, bW = xent_bounds(r, n, H, V, grad)
    for t, w, b in zip(got, (r["loss"], r["lse"], r["dX"], r["dW"]), (loss, loss, bX, bW)):
        within(host(t), w, b)


@pytest.mark.parametrize("dtype,grad", TYPES)
@pytest.mark.parametrize("H", [64, 128, 192, 256])
def test_xent_targets_at_every_place_of_a_tile(dtype, grad, H):
    """Each token the target of a row or two, then one token (at the edges of what a warp, a tile and the
    vocabulary hold) the target of all rows, and of a few in each 32."""
    n, V = 645, 517
    X, W, target, g = xent_inputs(n, H, V, dtype)
    check_bounds(dtype, grad, X, W, (np.arange(n) % V).astype(np.int32), g)
    for token in (0, 31, 32, 63, 64, 127, 128, 255, 256, 511, V - 1):
        target[:] = token
        check_bounds(dtype, grad, X, W, target, g)
    target = np.where(np.arange(n) % 13 == 0, 300, np.arange(n) % 7).astype(np.int32)
    check_bounds(dtype, grad, X, W, target, g)


@pytest.mark.parametrize("dtype,grad", TYPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_xent_of_logits_that_rise_or_fall_along_the_vocabulary(dtype, grad, sign):
    """Logits run over hundreds from the first token to the last: a running sum's reference has to move,
    or what comes later vanishes against it."""
    n, H, V = 140, 64, 1500
    rng = np.random.default_rng(11)
    W = rng.standard_normal((V, H)) * 0.05
    W[:, 0] = sign * np.linspace(-150.0, 150.0, V)
    X = rng.standard_normal((n, H)) * 0.1
    X[:, 0] = np.linspace(0.1, 2.0, n)
    target = rng.integers(0, V, n).astype(np.int32)
    g = (0.5 + rng.random(n)).astype(np.float32) / n
    check_bounds(dtype, grad, dev(X, dtype), dev(W, dtype), target, g)


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_xent_rows_left_out_may_hold_anything(dtype, grad):
    X, W, target, g = xent_inputs(333, 96, 210, dtype, 0.4)
    out = torch.from_numpy(target < 0).cuda()
    a = run_xent(dtype, X, W, target, g, grad)
    X[out] = float("nan")
    X[torch.nonzero(out)[::3, 0]] = float("inf")
    g = np.where(target < 0, np.float32("nan"), g)
    b = run_xent(dtype, X, W, target, g, grad)
    for u, v in zip(a, b):
        assert torch.equal(u, v)
    for u in a[:3]:
        assert torch.count_nonzero(u[out]) == 0


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_xent_with_no_row_left(dtype, grad):
    X, W, target, g = xent_inputs(200, 64, 150, dtype)
    target[:] = -1
    for t in run_xent(dtype, X, W, target, g, grad):
        assert torch.count_nonzero(t) == 0
    # and with no rows at all
    none = np.zeros(0, np.int32)
    for t in run_xent(dtype, X[:0], W, none, np.zeros(0, np.float32), grad):
        assert torch.count_nonzero(t) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_xent_accumulates_and_skips_what_is_not_asked(dtype):
    X, W, target, g = xent_inputs(190, 128, 140, dtype, 0.8)
    _, lse, dX, dW = run_xent(dtype, X, W, target, g, "f32")
    bX, bW = torch.randn_like(dX), torch.randn_like(dW)
    aX, aW = bX.clone(), bW.clone()
    run_xent(dtype, X, W, target, g, "f32", flags=L.BG_ACCUM, into=(aX, aW))
    # one more rounding of the sum, in either order
    assert (aX - (bX + dX)).abs().max() <= 4 * U * (bX.abs() + dX.abs()).max()
    assert (aW - (bW + dW)).abs().max() <= 4 * U * (bW.abs() + dW.abs()).max()
    t, gd = torch.from_numpy(target).cuda(), torch.from_numpy(g).cuda()
    ws = torch.empty(L.xent_workspace_bytes(dtype, 190, 128, 140, L.BG_OP_XENT_BWD), device="cuda",
                     dtype=torch.uint8)
    oX, oW = torch.empty_like(dX), torch.empty_like(dW)
    L.xent_bwd(dtype, X, W, t, lse, gd, "f32", oX, None, ws)
    L.xent_bwd(dtype, X, W, t, lse, gd, "f32", None, oW, ws)
    assert torch.equal(oX, dX) and torch.equal(oW, dW)


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_xent_gives_the_same_bits_again(dtype, grad):
    args = xent_inputs(3000, 64, 2000, dtype, 0.9)
    a, b = (run_xent(dtype, *args, grad) for _ in range(2))
    for u, v in zip(a, b):
        assert torch.equal(u, v)


def test_xent_reports_targets_past_the_vocabulary():
    X, W, target, g = xent_inputs(150, 64, 90, "bf16")
    target[[3, 140]] = [90, 2 ** 31 - 1]
    L.check_device()
    got = run_xent("bf16", X, W, target, g, "f32")
    with pytest.raises(L.BandGGNNError, match="site 131"):
        L.check_device()
    target[[3, 140]] = -1
    for u, v in zip(got, run_xent("bf16", X, W, target, g, "f32")):
        assert torch.equal(u, v)
    L.check_device()


@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** 50])
def test_xent_of_small_and_large_values(scale):
    """X small and W large by the same power of two, or the other way round: the logits are the same
    bits, dX and dW scale by it."""
    X, W, target, g = xent_inputs(140, 64, 300, "f32")
    a = run_xent("f32", X, W, target, g, "f32")
    b = run_xent("f32", X * scale, W / scale, target, g, "f32")
    r = ref.xent(host(X), host(W), target, g)
    loss, bX, bW = xent_bounds(r, 140, 64, 300, "f32")
    within(host(b[0]), r["loss"], loss)
    within(host(b[2]) * scale, r["dX"], bX)
    within(host(b[3]) / scale, r["dW"], bW)
    for u, v in zip(a[:2], b[:2]):
        assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("large", [1e6, 1e10, 1e15])
def test_xent_a_large_row_costs_the_others_nothing(dtype, large):
    """Rows are independent of one another: beside a few that are many times as large, and some as much
    smaller, the loss and dX of the others have the accuracy that they have among their likes."""
    n, H, V = 300, 64, 500
    X, W, target, g = xent_inputs(n, H, V, dtype)
    X[[7, 130, 299]] *= large
    X[[8, 131, 290]] /= large
    got = run_xent(dtype, X, W, target, g, "f32")
    rows = np.setdiff1d(np.arange(n), [7, 130, 299])
    only = np.full(n, -1, np.int32)
    only[rows] = target[rows]
    r = ref.xent(host(X), host(W), only, g)
    loss, bX, _ = xent_bounds(r, n, H, V, "f32")
    within(host(got[0])[rows], r["loss"][rows], loss[rows], "loss")
    within(host(got[1])[rows], r["lse"][rows], loss[rows], "lse")
    within(host(got[2])[rows], r["dX"][rows], bX[rows], "dX")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("large", [1e8, 1e10, 1e15, 1e30])
@pytest.mark.parametrize("V", [3, 500])
def test_xent_of_enormous_logits(dtype, large, V):
    """Logits far beyond what exp can tell apart: loss and lse are those of the largest one, to the
    precision of the logits, whatever their sign."""
    n, H = 260, 64
    X, W, target, g = xent_inputs(n, H, V, dtype)
    if V == 3:
        W, X[::2] = W.abs(), -X[::2].abs()  # every logit of these rows is negative
    X *= large
    t = torch.from_numpy(target).cuda()
    loss, lse = (torch.full((n,), float("nan"), device="cuda") for _ in range(2))
    ws = torch.empty(L.xent_workspace_bytes(dtype, n, H, V, L.BG_OP_XENT_FWD), device="cuda",
                     dtype=torch.uint8)
    L.xent_fwd(dtype, X, W, t, loss, lse, ws)
    r = ref.xent(host(X), host(W), target, g)
    tol = xent_bounds(r, n, H, V, "f32")[0]
    within(host(loss), r["loss"], tol, "loss")
    within(host(lse), r["lse"], tol, "lse")


@pytest.mark.parametrize("dtype,grad", TYPES)
@pytest.mark.parametrize("large", [1e6, 1e10, 1e20])
@pytest.mark.parametrize("H", [64, 128, 256])
def test_xent_gradients_beside_rows_of_enormous_logits(dtype, grad, large, H):
    """exp(z - lse) cannot be told from fp32 values of some 1e6 and more: such a row's probabilities are only
    kept within [0, 1].  So no element of dX or dW is more than each probability at its worst makes it, and the
    rest of dW, where those rows are left out, stands beside it."""
    n, V = 300, 500
    X, W, target, g = xent_inputs(n, H, V, dtype)
    far = [7, 130, 299]
    X[far] *= large
    g[130] = 0  # (a weight of 0 leaves nothing of an infinite one)
    got = run_xent(dtype, X, W, target, g, grad)
    only = target.copy()
    only[far] = -1
    r = ref.xent(host(X), host(W), only, g)
    loss, bX, bW = xent_bounds(r, n, H, V, grad)
    near = np.setdiff1d(np.arange(n), far)
    within(host(got[2])[near], r["dX"][near], bX[near], "dX")
    # a far row: every probability from 0 to 1, its target's less 1; results rounded
    x, w = np.abs(host(X)), np.abs(host(W))
    more = 1 + 2.0 ** -7
    assert (np.abs(host(got[2])[far]) <= more * g[far][:, None] * w.sum(0) + bX[far]).all()
    within(host(got[3]), r["dW"], bW + more * ((g[far][:, None] * x[far]).sum(0)) + 2.0 ** -7 * np.abs(r["dW"]), "dW")
    # a token's row of dW takes nothing from a far row whose logit is far below its largest
    z = host(X)[far] @ host(W).T
    low = (z < z.max(1, keepdims=True) - 0.01 * np.abs(z).max(1, keepdims=True)).all(0)
    low[target[far]] = False
    assert low.sum() > V // 2
    floor = 2.0 ** -37 * (g[:, None] * x).max() if grad == "f32" else 0
    within(host(got[3])[low], r["dW"][low], bW[low] + n * floor, "dW of tokens that far rows do not reach")


def test_xent_of_a_table_with_one_large_row():
    """An element of W is off by 2^-39 of W's largest at most, a logit by that times the sum of its state:
    rows that the large token does not dominate keep a loss of that accuracy."""
    n, H, V = 300, 64, 500
    X, W, target, g = xent_inputs(n, H, V, "f32")
    W[3] *= 1e8
    target[target == 3] = 4
    z = host(X) @ host(W).T
    rows = np.flatnonzero(z[:, 3] < -1e3)
    assert rows.size > n // 4
    got = run_xent("f32", X, W, target, g, "f32")
    r = ref.xent(host(X), host(W), target, g)
    zabs = (np.abs(host(X[rows])) @ np.delete(np.abs(host(W)), 3, 0).T).max()
    dz = (2 * H * U + 2.0 ** -21) * zabs + 2.0 ** -39 * np.abs(host(W)).max() * np.abs(host(X[rows])).sum(1)
    tol = 2 * dz + 2.0 ** -20 * (1 + np.abs(r["lse"][rows]))
    within(host(got[0])[rows], r["loss"][rows], tol, "loss")
    within(host(got[1])[rows], r["lse"][rows], tol, "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_xent_gradient_against_differences(dtype):
    """Directional differences of the forward itself, over states and table.  With step e along a
    direction whose logits move by at most m, the central difference is off by e^2 m^3 / 6 of the
    weights' sum, and by the loss's rounding over e."""
    n, H, V = 96, 64, 200
    X, W, target, g = xent_inputs(n, H, V, dtype)
    rng = np.random.default_rng(3)
    r = ref.xent(host(X), host(W), target, g)
    _, _, dX, dW = run_xent(dtype, X, W, target, g, "f32")
    # differences are taken in fp32 on the values the gradient was taken at
    Xf, Wf = X.float(), W.float()
    for which, d in (("X", dX), ("W", dW)):
        D = rng.standard_normal(tuple(d.shape))
        Dd = dev(D, "f32")
        move = host(Dd) @ host(Wf).T if which == "X" else host(Xf) @ host(Dd).T
        m = 2 * np.abs(move).max()
        e = 0.02 / m
        f = []
        for s in (e, -e):
            args = (Xf + s * Dd, Wf) if which == "X" else (Xf, Wf + s * Dd)
            f.append(float((host(run_xent("f32", *args, target, g, "f32")[0]) * g).sum()))
        got = float((host(d) * host(Dd)).sum())
        want = (f[0] - f[1]) / (2 * e)
        loss, bX, bW = xent_bounds(r, n, H, V, "f32")
        # X + e D itself is rounded to fp32: a logit moves by u of its magnitude
        tol = g.sum() * ((e * m) ** 2 * m / 6 + (loss.max() + 2 * U * r["zabs"]) / e)
        assert abs(got - want) <= tol, (which, got, want, tol)


def test_xent_past_32_bits_of_elements():
    """n H just over 2^31 with few labelled rows, the last ones among them."""
    n, H, V = (1 << 23) + 70, 256, 5
    X = torch.zeros(n, H, device="cuda", dtype=torch.bfloat16)
    target = np.full(n, -1, np.int32)
    at = np.array([0, 5, 1 << 20, (1 << 23) - 1, n - 2, n - 1])
    target[at] = [0, 4, 2, 3, 1, 0]
    small, W, _, _ = xent_inputs(6, H, V, "bf16")
    X[torch.from_numpy(at).cuda()] = small
    g = np.ones(n, np.float32)
    loss, lse, dX, dW = run_xent("bf16", X, W, target, g, "bf16")
    r = ref.xent(host(small), host(W), target[at], g[at])
    b, bX, bW = xent_bounds(r, 6, H, V, "bf16")
    pick = torch.from_numpy(at).cuda()
    within(host(loss[pick]), r["loss"], b)
    within(host(dX[pick]), r["dX"], bX)
    within(host(dW), r["dW"], bW)
    assert int(torch.count_nonzero(loss)) == int(np.count_nonzero(host(loss[pick])))
    dX[pick] = 0
    assert torch.count_nonzero(dX) == 0


@pytest.mark.parametrize("which", ["dX", "dW"])
def test_xent_bf16_gradients_of_long_sums(which):
    """Millions of terms of one sign to an element.  The tensor core drops what does not fit its fp32
    accumulator, all in one direction: left there, sums like these are 4% low.  They have to leave it long
    before that.

    All logits are 0, so that every probability is 1 / V, and V is such that 1 / V is within 2^-16 of a
    bf16 number p: an element is p times a column's sum.  Rounding the result to bf16 is off by up to 2^-8
    either way; over 256 columns of random size the mean of that is below 6 x 2^-8 / sqrt(3 x 256).  2^-13
    on top is left for what is lost before a sum leaves the accumulator."""
    H = 256
    rows, V = (19456, 8421505) if which == "dX" else (1 << 23, 16448)
    many = V if which == "dX" else rows  # the side that is summed over
    p = float(torch.tensor(1.0 / V).to(torch.bfloat16).double())
    assert abs(p * V - 1) < 2.0 ** -15
    gen = torch.Generator(device="cuda").manual_seed(1)
    size = 1 + torch.rand(H, generator=gen, device="cuda")
    side = torch.empty(many, H, device="cuda", dtype=torch.bfloat16)
    total = torch.zeros(H, device="cuda", dtype=torch.float64)
    for piece in side.split(1 << 20):
        piece.copy_((1 + torch.rand(piece.shape, generator=gen, device="cuda")) * size)
    side[0] = 0  # (the target's row of W)
    for piece in side.split(1 << 20):
        total += piece.double().sum(0)
    none = torch.zeros(rows if which == "dX" else V, H, device="cuda", dtype=torch.bfloat16)
    X, W = (none, side) if which == "dX" else (side, none)
    target = torch.zeros(rows, device="cuda", dtype=torch.int32)
    lse = torch.full((rows,), float(np.log(V)), device="cuda")
    g = torch.ones(rows, device="cuda")
    out = torch.full_like(none, float("nan"))
    ws = torch.empty(L.xent_workspace_bytes("bf16", rows, H, V, L.BG_OP_XENT_BWD), device="cuda",
                     dtype=torch.uint8)
    dX, dW = (out, None) if which == "dX" else (None, out)
    L.xent_bwd("bf16", X, W, target, lse, g, "bf16", dX, dW, ws)
    L.check_device()
    want = host(total) * p
    for at in (1, len(out) // 2, len(out) - 1):
        off = host(out[at]) / want - 1
        assert np.abs(off).max() < 2.0 ** -8 + 2.0 ** -12
        assert abs(off.mean()) < 6 * 2.0 ** -8 / np.sqrt(3 * H) + 2.0 ** -13, off.mean()


# ------------------------------------------------------------------------------ streams


def test_token_operators_run_on_the_stream_they_are_given():
    """Inputs made on a side stream, operators given that stream, results read after it alone; and the
    same calls captured in a CUDA graph and replayed on new values."""
    n, H, V = 700, 64, 333
    X, W, target, g = xent_inputs(n, H, V, "bf16", 0.8)
    want = run_xent("bf16", X, W, target, g, "f32")
    st = torch.cuda.Stream()
    t, gd = torch.from_numpy(target).cuda(), torch.from_numpy(g).cuda()
    ws = torch.empty(max(L.xent_workspace_bytes("bf16", n, H, V, op)
                         for op in (L.BG_OP_XENT_FWD, L.BG_OP_XENT_BWD)), device="cuda",
                     dtype=torch.uint8)
    ews = torch.empty(L.embed_workspace_bytes(n, H, V), device="cuda", dtype=torch.uint8)
    x2 = torch.zeros_like(X)
    outs = [torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"),
            torch.zeros(n, H, device="cuda"), torch.zeros(V, H, device="cuda")]
    dE = torch.zeros(V, H, device="cuda")

    def calls(stream):
        L.dropout_fwd("bf16", x2, x2, 0.0, SEED, CALL, stream=stream)
        L.xent_fwd("bf16", x2, W, t, outs[0], outs[1], ws, stream=stream)
        L.xent_bwd("bf16", x2, W, t, outs[1], gd, "f32", outs[2], outs[3], ws, stream=stream)
        L.embed_bwd(t, outs[2], dE, ews, stream=stream)

    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        x2.copy_(X)
    calls(st)
    st.synchronize()
    for u, v in zip(outs, want):
        assert torch.equal(u, v)
    first = dE.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        calls(None)
    for o in outs + [dE]:
        o.zero_()
    x2.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.count_nonzero(outs[2]) and not torch.equal(outs[2], want[2])
    x2.copy_(X)
    graph.replay()
    torch.cuda.synchronize()
    for u, v in zip(outs, want):
        assert torch.equal(u, v)
    assert torch.equal(dE, first)


FIRST_CALLS = """
import torch
from paper_1906_11786_gb300 import lib as L
n, H, V = 500, 64, 300
gen = torch.Generator(device="cuda").manual_seed(1)
X, W, dout = (torch.randn(m, H, device="cuda", generator=gen) for m in (n, V, n))
t = torch.randint(0, V, (n,), device="cuda", generator=gen, dtype=torch.int32)
g = torch.ones(n, device="cuda")
ws = torch.empty(max([L.embed_workspace_bytes(n, H, V)] +
                     [L.xent_workspace_bytes("f32", n, H, V, op)
                      for op in (L.BG_OP_XENT_FWD, L.BG_OP_XENT_BWD)]), device="cuda",
                 dtype=torch.uint8)
outs = [torch.zeros(*s, device="cuda") for s in ((n, H), (V, H), (n,), (n,), (n, H), (V, H))]
out, dtable, loss, lse, dX, dW = outs

def calls():
    L.embed_fwd("f32", t, W, out, p=0.1, seed=3, call=4)
    L.embed_bwd(t, dout, dtable, ws)
    L.xent_fwd("f32", X, W, t, loss, lse, ws)
    L.xent_bwd("f32", X, W, t, lse, g, "f32", dX, dW, ws)

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls()
graph.replay()
torch.cuda.synchronize()
L.check_device()
replayed = [o.clone() for o in outs]
for o in outs:
    o.zero_()
calls()
torch.cuda.synchronize()
L.check_device()
assert all(torch.equal(a, b) and torch.count_nonzero(a) for a, b in zip(replayed, outs))
print("captured")
"""


def test_the_first_token_calls_of_a_process_can_be_captured():
    """No plan comes before them, so that a process may capture its very first call to the library."""
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, timeout=300,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]
