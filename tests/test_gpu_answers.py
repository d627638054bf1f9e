"""GPU parity of the operators that answer with a vocabulary (logits, their adjustment, the largest of
each row) against plain implementations, at the sizes, alignments, masks and values where they can go wrong.

u = 2^-24 is half the gap of fp32.  Adjusted logits are defined operation by operation in fp32, so they, and
with them the chosen tokens, are compared bit for bit; what is summed has a bound derived beside it.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import answer_ref as ref
from gpu_common import ensure_built
from paper_1906_11786_gb300 import _binding as L

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = 2.0 ** -8  # rounding to bf16, relative
TD = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()


def dev(x, dtype="f32"):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(TD[dtype]).cuda()


def ints(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(x, dtype)).cuda()


def host(t):
    return t.double().cpu().numpy()


def rows(n, V, pad, dtype, fill=float("nan")):
    """([n, V] view with rows V + pad apart, the buffer under it, filled)"""
    buf = torch.full((n, V + pad), fill, device="cuda", dtype=TD[dtype])
    return buf[:, :V], buf


def within(got, want, tol, what=""):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape
    assert np.all(np.isfinite(got)), f"{what}: not finite"
    over = np.abs(got - want) - tol
    assert over.size == 0 or over.max() <= 0, \
        f"{what}: {np.abs(got - want).flat[over.argmax()]:.3e} off at {over.argmax()}"


# ------------------------------------------------------------------------------ logits


def logits_tolerance(X, W, dtype, out):
    """A step of 16 products loses at most 4 u of the accumulator (one sign; it truncates), which stays below
    S = sum |x| |w|: H / 16 steps, three times as many for two terms, of which two thirds at 2^-11 of S.
    Two terms: each operand is off by 2^-22 of itself, and below 2^-17 of its row's largest by 2^-39 of that;
    low x low is left out: 2^-22 of the product."""
    X, W = np.abs(np.asarray(X, np.float64)), np.abs(np.asarray(W, np.float64))
    S, H = X @ W.T, X.shape[1]
    tol = 4 * U * (H // 16 + 1) * S
    if dtype == "f32":
        tol = tol * 1.01 + 3 * 2.0 ** -22 * S
        tol += 2.0 ** -39 * (X.max(1, keepdims=True) * W.sum(1)[None] + X.sum(1, keepdims=True) * W.max(1)[None])
    return tol


def check_logits(n, H, V, dtype, out, pad=0, seed=0, X=None, W=None):
    rng = np.random.default_rng(seed)
    X = dev(rng.standard_normal((n, H)) if X is None else X, dtype)
    W = dev(rng.standard_normal((V, H)) * 0.3 if W is None else W, dtype)
    Z, buf = rows(n, V, pad, out, 7.0)
    need = L.logits_workspace_bytes(dtype, n, H, V)
    ws = torch.full((need,), 0xFF, device="cuda", dtype=torch.uint8) if need else None
    L.logits_fwd(dtype, X, W, out, Z, ws)
    L.check_device()
    want = host(X) @ host(W).T
    tol = logits_tolerance(host(X), host(W), dtype, out) + 2.0 ** -126
    if out == "bf16":
        tol = tol * 1.01 + HALF * 1.01 * np.abs(want)
    within(host(Z), want, tol, "Z")
    assert bool((buf[:, V:] == 7.0).all()), "the elements between rows were written"
    return Z


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,H,V", [(1, 32, 1), (1, 128, 32000), (2, 96, 129), (15, 64, 127), (16, 160, 128),
                                   (17, 256, 1000), (33, 224, 50), (128, 128, 513), (129, 32, 700),
                                   (255, 64, 255), (256, 256, 300), (257, 192, 4001), (1000, 256, 3001)])
def test_logits(n, H, V, dtype):
    check_logits(n, H, V, dtype, "f32", seed=n)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [0, 1, 17])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_rows_of_any_length_and_type(dtype, pad, out):
    check_logits(301, 64, 777, dtype, out, pad=pad)


@pytest.mark.parametrize("dtype,n,H,V", [("bf16", 40001, 64, 2000), ("f32", 20000, 96, 3000),
                                         ("bf16", 700, 256, 49999)])
def test_logits_of_many_tiles(dtype, n, H, V):
    check_logits(n, H, V, dtype, "f32", seed=3)


def test_logits_of_rows_of_mixed_magnitude():
    """A row's logits depend on no other row: each row of X and of W has a scale of its own, from 2^-80 to 2^40
    (products from 2^-160, which are 0, to 2^80)."""
    rng = np.random.default_rng(5)
    n, H, V = 70, 64, 300
    X = rng.standard_normal((n, H)) * 2.0 ** rng.integers(-80, 41, (n, 1))
    W = rng.standard_normal((V, H)) * 2.0 ** rng.integers(-80, 41, (V, 1))
    X[7], W[11] = 0.0, 0.0
    check_logits(n, H, V, "f32", "f32", X=X, W=W)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_of_rows_that_are_not_finite_stay_theirs(dtype):
    rng = np.random.default_rng(6)
    n, H, V = 300, 64, 400
    X, W = rng.standard_normal((n, H)), rng.standard_normal((V, H))
    X[5, 3], X[299, 0], W[17, 9] = np.nan, np.inf, -np.inf
    Z, _ = rows(n, V, 0, "f32")
    need = L.logits_workspace_bytes(dtype, n, H, V)
    L.logits_fwd(dtype, dev(X, dtype), dev(W, dtype), "f32", Z,
                 torch.empty(need, device="cuda", dtype=torch.uint8) if need else None)
    bad = np.zeros((n, V), bool)
    bad[5], bad[299], bad[:, 17] = True, True, True
    assert np.array_equal(np.isfinite(host(Z)), ~bad)


# ------------------------------------------------------------------------------ adjustment


def constraints(n, V, seed, bias=True, masks=3, history=40):
    """kwargs of answer_ref.adjusted and the LogitAdjust of the same."""
    rng = np.random.default_rng(seed)
    kw, own = {}, {}
    if bias:
        kw["bias"] = rng.standard_normal(V).astype(np.float32)
        kw["bias"][rng.random(V) < 0.05] = -np.inf
        own["bias"] = dev(kw["bias"])
    if masks:
        kw["allowed"] = rng.random((masks, V)) < rng.choice([0.02, 0.5, 0.97], (masks, 1))
        if masks > 2:
            kw["allowed"][0] = False  # leaves nothing
        kw["mask_row"] = rng.integers(-1, masks, n)
        own["mask"] = torch.from_numpy(ref.pack_mask(kw["allowed"])).cuda()
        own["mask_row"] = ints(kw["mask_row"])
    if history:
        kw["history"] = [rng.integers(-1, V, rng.integers(0, history + 1)) % (V // 3 + 1) - (rng.random() < 0.3)
                         for _ in range(n)]
        kw["penalty"] = np.stack([1 + rng.random(n), rng.standard_normal(n), rng.random(n)], 1).astype(np.float32)
        off = np.concatenate([[0], np.cumsum([len(h) for h in kw["history"]])])
        own["history"] = ints(np.concatenate(kw["history"]) if off[-1] else np.zeros(0))
        own["history_off"], own["penalty"] = ints(off, np.int64), dev(kw["penalty"])
    return kw, L.LogitAdjust(**own)


def bits(t):
    """The bits of a tensor, NaN as one value."""
    t = torch.where(torch.isnan(t), torch.full_like(t, float("nan")), t)
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).cpu().numpy()


SHAPES = [(1, 1), (1, 32000), (3, 31), (4, 33), (5, 129), (2, 8191), (3, 8192), (7, 8193), (9, 20001), (300, 513)]


@pytest.mark.parametrize("parts", [dict(), dict(bias=False, masks=0), dict(bias=False, history=0),
                                   dict(masks=0, history=0), dict(history=0), dict(bias=False, masks=1),
                                   dict(bias=False, masks=0, history=0)])
@pytest.mark.parametrize("dtype,pad", [("f32", 0), ("f32", 3), ("bf16", 0), ("bf16", 5)])
def test_adjust_is_bit_exact(dtype, pad, parts):
    for n, V in SHAPES:
        rng = np.random.default_rng(n * V)
        Z, buf = rows(n, V, pad, dtype, 7.0)
        Z.copy_(dev(rng.standard_normal((n, V)) * 3, dtype))
        kw, adjust = constraints(n, V, n + V, **parts)
        out, obuf = rows(n, V, (pad + 2) % 5, dtype, 9.0)
        before = buf.clone()
        L.logits_adjust(dtype, Z, out, adjust)
        L.check_device()
        want = torch.from_numpy(ref.adjusted(host(Z), **kw)).to(TD[dtype]).cuda()
        assert np.array_equal(bits(out), bits(want)), (n, V)
        assert bool((obuf[:, V:] == 9.0).all()) and torch.equal(buf, before)
        L.logits_adjust(dtype, Z, Z, adjust)  # in place
        assert np.array_equal(bits(Z), bits(want)), (n, V, "in place")
        assert bool((buf[:, V:] == 7.0).all())


def test_adjust_of_values_that_are_not_finite():
    """A masked place is -inf whatever stood there; elsewhere infinities and NaN go the way of the formula."""
    n, V = 4, 1001
    rng = np.random.default_rng(1)
    z = rng.standard_normal((n, V)).astype(np.float32)
    z[:, ::7], z[:, 1::7], z[:, 2::7], z[:, 3::7] = np.nan, np.inf, -np.inf, np.finfo(np.float32).min
    kw, adjust = constraints(n, V, 2)
    out = torch.empty(n, V, device="cuda")
    L.logits_adjust("f32", dev(z), out, adjust)
    assert np.array_equal(bits(out), bits(torch.from_numpy(ref.adjusted(z, **kw)).cuda()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_penalties_of_long_and_repetitive_histories(dtype):
    """Histories of no, one, and 200000 tokens, of one token alone and of tokens at a segment's ends."""
    V = 30000
    rng = np.random.default_rng(3)
    history = [np.zeros(0, int), np.array([V - 1]), rng.integers(0, V, 200000), np.full(70001, 8191),
               np.array([0, 8191, 8192, 16383, 16384, V - 1, 8192, -5, 0])]
    n = len(history)
    penalty = np.stack([np.full(n, 1.3), np.full(n, 0.25), np.full(n, 0.001)], 1).astype(np.float32)
    z = dev(rng.standard_normal((n, V)), dtype)
    off = np.concatenate([[0], np.cumsum([len(h) for h in history])])
    adjust = L.LogitAdjust(history=ints(np.concatenate(history)), history_off=ints(off, np.int64),
                           penalty=dev(penalty))
    want = ref.adjusted(host(z), history=history, penalty=penalty)
    out = torch.empty_like(z)
    L.logits_adjust(dtype, z, out, adjust)
    assert np.array_equal(bits(out), bits(torch.from_numpy(want).to(TD[dtype]).cuda()))
    check_top(z, 9, dtype, adjust, want)


def test_a_mask_for_each_row_and_one_for_all():
    n, V = 6, 100
    rng = np.random.default_rng(4)
    z = rng.standard_normal((n, V)).astype(np.float32)
    for masks in (1, n, n + 3):
        allowed = rng.random((masks, V)) < 0.5
        out = torch.empty(n, V, device="cuda")
        L.logits_adjust("f32", dev(z), out, L.LogitAdjust(mask=torch.from_numpy(ref.pack_mask(allowed)).cuda()))
        assert np.array_equal(bits(out), bits(torch.from_numpy(ref.adjusted(z, allowed=allowed)).cuda()))


def test_bad_tokens_masks_and_offsets_are_reported_and_skipped():
    n, V = 3, 50
    z = np.random.default_rng(7).standard_normal((n, V)).astype(np.float32)
    out, ids = torch.empty(n, V, device="cuda"), torch.empty(n, 2, device="cuda", dtype=torch.int32)
    vals = torch.empty(n, 2, device="cuda")
    pen = np.full((n, 3), 1.5, np.float32)

    def both(adjust, site, want):
        L.logits_adjust("f32", dev(z), out, adjust)
        with pytest.raises(L.BandGGNNError, match=f"site {site}"):
            L.check_device()
        assert np.array_equal(bits(out), bits(torch.from_numpy(want).cuda()))
        L.logits_top("f32", dev(z), vals, ids, None, adjust)
        with pytest.raises(L.BandGGNNError, match=f"site {site}"):
            L.check_device()
        assert np.array_equal(ids.cpu().numpy(), ref.top(want, 2)[1])
        L.check_device()

    both(L.LogitAdjust(history=ints([1, V, 2]), history_off=ints([0, 2, 2, 3], np.int64), penalty=dev(pen)),
         132, ref.adjusted(z, history=[[1], [], [2]], penalty=pen))
    allowed = np.arange(V)[None] % 2 == np.arange(2)[:, None]
    both(L.LogitAdjust(mask=torch.from_numpy(ref.pack_mask(allowed)).cuda(), mask_row=ints([1, 2, 0])),
         133, ref.adjusted(z, allowed=allowed, mask_row=[1, -1, 0]))
    for off, kept in (([0, 2, 1, 3], [[1, 5], [], [5, 2]]), ([0, 1, 1, 4], [[1], [], []]), ([-1, 2, 2, 3], [[], [], [2]])):
        both(L.LogitAdjust(history=ints([1, 5, 2]), history_off=ints(off, np.int64), penalty=dev(pen)), 134,
             ref.adjusted(z, history=kept, penalty=pen))


# ------------------------------------------------------------------------------ largest logits


def lse_tolerance(z, V):
    """exp2's 2^-22, the rounding of its argument c z - m (c = log2 e rounded: u |z|, and u of the difference,
    at most 2 |z|), the sums (no more than V / 256 + 40 additions deep, u each), the result's roundings (4 u)."""
    big = np.where(np.isfinite(z), np.abs(np.asarray(z, np.float64)), 0).max(1)
    return 2.0 ** -22 + U * (V / 256 + 40) + 10 * U * big


def check_top(Z, K, dtype, adjust, adjusted):
    n, V = Z.shape
    vals = torch.full((n, K), 5.0, device="cuda")
    ids = torch.full((n, K), 77, device="cuda", dtype=torch.int32)
    lse = torch.full((n,), 5.0, device="cuda")
    L.logits_top(dtype, Z, vals, ids, lse, adjust)
    L.check_device()
    wv, wi, wl = ref.top(adjusted, K)
    assert np.array_equal(ids.cpu().numpy(), wi)
    assert np.array_equal(vals.cpu().numpy(), wv)
    got, some = host(lse), np.isfinite(wl)
    assert np.array_equal(got[~some], wl[~some], equal_nan=True)
    if some.any():
        within(got[some], wl[some], lse_tolerance(adjusted[some], V), "lse")
    only = torch.full_like(ids, 77)
    L.logits_top(dtype, Z, vals, only, None, adjust)
    assert torch.equal(only, ids)


@pytest.mark.parametrize("dtype,pad", [("f32", 0), ("f32", 1), ("bf16", 0), ("bf16", 3)])
@pytest.mark.parametrize("K", [1, 5, 64, 128])
def test_top(K, dtype, pad):
    for n, V in SHAPES + [(1, 5000), (200, 30001), (77, 12000), (400, 9001)]:
        rng = np.random.default_rng(V)
        Z, _ = rows(n, V, pad, dtype)
        Z.copy_(dev(rng.standard_normal((n, V)) * 3, dtype))
        check_top(Z, K, dtype, None, host(Z).astype(np.float32))


@pytest.mark.parametrize("parts", [dict(), dict(bias=False, masks=0), dict(bias=False, history=0),
                                   dict(masks=0, history=0), dict(history=0), dict(bias=False, masks=1),
                                   dict(masks=0)])
@pytest.mark.parametrize("dtype,pad", [("f32", 0), ("bf16", 1)])
def test_top_of_adjusted_logits(dtype, pad, parts):
    for n, V in SHAPES + [(170, 20001)]:
        rng = np.random.default_rng(V)
        Z, _ = rows(n, V, pad, dtype)
        Z.copy_(dev(rng.standard_normal((n, V)) * 3, dtype))
        kw, adjust = constraints(n, V, n + V, **parts)
        check_top(Z, 16, dtype, adjust, ref.adjusted(host(Z), **kw))


@pytest.mark.parametrize("n", [2, 310])
@pytest.mark.parametrize("kind", ["constant", "rising", "falling", "two values", "steps", "zeros of both signs",
                                  "one answer", "none", "not finite"])
def test_top_of_rows_made_to_be_hard(kind, n):
    """Ties without end, every logit larger than the last, and rows with nothing to answer."""
    V = 20003
    v = np.arange(V)
    z = {"constant": np.full(V, 1.5), "rising": v / 64.0, "falling": -v / 64.0,
         "two values": np.where(v % 3 == 0, 2.0, 1.0), "steps": (v // 500) * 0.5,
         "zeros of both signs": np.where(v % 2 == 0, -0.0, 0.0), "one answer": np.where(v == 12345, -3e30, -np.inf),
         "none": np.full(V, -np.inf),
         "not finite": np.where(v % 1000 == 7, np.inf, np.where(v % 1000 == 8, np.nan, -v))}[kind]
    z = np.tile(z.astype(np.float32), (n, 1))
    for K in (1, 100, 128):
        check_top(dev(z), K, "f32", None, z)


def test_top_from_rows_beyond_32_bit_offsets():
    """Rows at element offsets past 2^32, in a buffer of which only they are used."""
    n, V, ld = 3, 700, (1 << 31) - 8
    buf = torch.empty((n - 1) * ld + V, device="cuda", dtype=torch.bfloat16)
    Z = buf.as_strided((n, V), (ld, 1))
    z = np.random.default_rng(8).standard_normal((n, V))
    Z.copy_(dev(z, "bf16"))
    kw, adjust = constraints(n, V, 1)
    check_top(Z, 7, "bf16", adjust, ref.adjusted(host(Z), **kw))
    L.logits_adjust("bf16", Z, Z, adjust)
    assert np.array_equal(bits(Z), bits(torch.from_numpy(ref.adjusted(z_bf16(z), **kw)).to(torch.bfloat16).cuda()))


def z_bf16(z):
    return torch.from_numpy(np.asarray(z, np.float32)).to(torch.bfloat16).double().numpy()
