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
                                   (255, 64, 255), (256, 256, 300), (257, 192, 4001), (1000, 256, 3001), (3, 96, 1001), (4, 32, 999),
                                   (5, 224, 130), (4, 256, 5000), (3, 160, 33)])
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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 3, 4, 5, 40])
@pytest.mark.parametrize("H", [32, 96, 160, 256])
def test_logits_of_infinite_elements_do_not_depend_on_the_number_of_rows(H, n, dtype):
    """fp32: NaN; bf16: what products and sum are; and infinite where finite elements' sum overflows."""
    V = 300
    rng = np.random.default_rng(H + n)
    X, W = rng.standard_normal((n, H)), rng.standard_normal((V, H))
    X[n - 1, H - 1] = np.inf
    W[17, 9], W[33, 1], W[40, :], W[299, 0] = -np.inf, np.nan, 0.0, np.inf
    if n > 1:
        X[0, :], W[5, :], W[6, :] = 2.0 ** 100, 2.0 ** 100, -2.0 ** 100
    Z, _ = rows(n, V, 1, "f32")
    need = L.logits_workspace_bytes(dtype, n, H, V)
    L.logits_fwd(dtype, dev(X, dtype), dev(W, dtype), "f32", Z,
                 torch.empty(need, device="cuda", dtype=torch.uint8) if need else None)
    x, w = host(dev(X, dtype)), host(dev(W, dtype))
    with np.errstate(all="ignore"):
        want = (x[:, None] * w[None]).sum(2)
        if dtype == "f32":
            want[~np.isfinite(x).all(1)] = np.nan
            want[:, ~np.isfinite(w).all(1)] = np.nan
        want = want.astype(np.float32)
    got = Z.cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.where(np.isinf(got), got, 0), np.where(np.isinf(want), want, 0))


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_logits_and_their_readers_from_the_middle_of_a_sector(out, pad):
    """Pointers are aligned to 16 bytes, not to the 32 of a sector."""
    n, H, V = 70, 64, 900
    rng = np.random.default_rng(0)
    X, W = dev(rng.standard_normal((n, H)), "bf16"), dev(rng.standard_normal((V, H)) * 0.3, "bf16")
    lead = 16 // TD[out].itemsize
    buf = torch.full((lead + n * (V + pad),), 7.0, device="cuda", dtype=TD[out])
    Z = buf[lead:].view(n, V + pad)[:, :V]
    assert Z.data_ptr() % 32 == 16
    L.logits_fwd("bf16", X, W, out, Z)
    want = host(X) @ host(W).T
    tol = logits_tolerance(host(X), host(W), "bf16", out)
    within(host(Z), want, tol * 1.01 + HALF * 1.01 * np.abs(want) if out == "bf16" else tol)
    assert bool((buf[:lead] == 7.0).all())
    kw, adjust = constraints(n, V, 3)
    adj = ref.adjusted(host(Z), **kw)
    check_top(Z, 17, out, adjust, adj)
    L.logits_adjust(out, Z, Z, adjust)
    assert np.array_equal(bits(Z), bits(torch.from_numpy(adj).to(TD[out]).cuda()))
    assert bool((buf[:lead] == 7.0).all())


def test_logits_past_32_bits_of_elements():
    """86001 x 50001 logits (4.3 10^9); rows all along, and the tokens at both ends, against 64 bits."""
    n, H, V = 86001, 32, 50001
    gen = torch.Generator(device="cuda").manual_seed(5)
    X, W = (torch.randn(m, H, device="cuda", generator=gen).to(torch.bfloat16) for m in (n, V))
    Z = torch.empty(n, V, device="cuda", dtype=torch.bfloat16)
    L.logits_fwd("bf16", X, W, "bf16", Z)
    L.check_device()
    for i in list(range(0, n, 9001)) + [n - 2, n - 1, 42949, 42950]:
        want = host(X[i:i + 1]) @ host(W).T
        tol = logits_tolerance(host(X[i:i + 1]), host(W), "bf16", "bf16")
        within(host(Z[i:i + 1]), want, tol * 1.01 + HALF * 1.01 * np.abs(want))
    top = torch.empty(n, 3, device="cuda")
    ids = torch.empty(n, 3, device="cuda", dtype=torch.int32)
    L.logits_top("bf16", Z, top, ids)
    assert torch.equal(top.max(1).values, Z.max(1).values.float())
    assert torch.equal(Z.gather(1, ids.long()).float(), top)


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


@pytest.mark.parametrize("n,V", [(37, 8191), (37, 8193), (37, 16385), (130, 20001), (700, 20001), (2500, 9001),
                                 (33, 70001)])
@pytest.mark.parametrize("dtype,pad", [("f32", 0), ("f32", 2), ("bf16", 0), ("bf16", 1), ("bf16", 2), ("bf16", 4)])
@pytest.mark.parametrize("parts", ["all", "bias", "bias and mask", "bias and histories", "long histories"])
def test_adjust_of_rows_over_several_runs_of_biases(parts, dtype, pad, n, V):
    """Rows that begin anywhere in 16 bytes share runs of 8192 biases; histories follow in a launch of their own,
    except in place, and long ones do the row again."""
    rng = np.random.default_rng(n + V)
    kw = {"bias": rng.standard_normal(V).astype(np.float32)}
    if parts in ("all", "bias and mask"):
        kw["allowed"], kw["mask_row"] = rng.random((3, V)) < 0.7, rng.integers(-1, 3, n)
    if parts not in ("bias", "bias and mask"):
        most = 40 if parts == "all" else 300
        kw["history"] = [rng.integers(0, V, 1537 + i if parts == "long histories" and i % 31 == 5 else
                                      rng.integers(0, most)) for i in range(n)]
        for h in kw["history"][:3]:
            h[:2] = (0, V - 1)[:len(h)]
        kw["penalty"] = np.stack([1 + rng.random(n), rng.standard_normal(n), rng.random(n)], 1).astype(np.float32)
    Z, buf = rows(n, V, pad, dtype, 7.0)
    Z.copy_(3 * torch.randn(n, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(V)))
    adjust = repeated(kw, 1)
    want = torch.from_numpy(ref.adjusted(Z.float().cpu().numpy(), **kw)).to(TD[dtype]).cuda()
    for other in (0, 1):  # of the same distance between rows, and of another
        out, obuf = rows(n, V, pad + other, dtype, 9.0)
        L.logits_adjust(dtype, Z, out, adjust)
        L.check_device()
        assert torch.equal(out, want) and bool((obuf[:, V:] == 9.0).all())
    L.logits_adjust(dtype, Z, Z, adjust)
    assert torch.equal(Z, want) and bool((buf[:, V:] == 7.0).all())


@pytest.mark.parametrize("V,pad", [(32769, 0), (40001, 2), (49999, 0)])
@pytest.mark.parametrize("parts", ["bias", "bias and mask", "all", "long histories"])
def test_adjust_of_many_long_rows_at_odd_places(parts, V, pad):
    """bf16 rows from 2^27 elements on share their biases; the same rows again and again begin at every place."""
    distinct, times = 41, 103
    assert V >= 32768 and distinct * times * V >= 1 << 27 and (V + pad) % 2
    rng = np.random.default_rng(V)
    kw = {"bias": rng.standard_normal(V).astype(np.float32)}
    if parts in ("all", "bias and mask"):
        kw["allowed"], kw["mask_row"] = rng.random((3, V)) < 0.7, rng.integers(-1, 3, distinct)
    if parts in ("all", "long histories"):
        kw["history"] = [np.concatenate([[0, V - 1, 8191, 8192], rng.integers(0, V, 1533 + i if parts != "all" and i % 9 == 5
                                                                              else rng.integers(0, 300))])
                         for i in range(distinct)]
        kw["penalty"] = np.stack([1 + rng.random(distinct), rng.standard_normal(distinct), rng.random(distinct)],
                                 1).astype(np.float32)
    one = dev(rng.standard_normal((distinct, V)) * 3, "bf16")
    Z, buf = rows(distinct * times, V, pad, "bf16", 7.0)
    Z.copy_(one.repeat(times, 1))
    adjust = repeated(kw, times)
    want = torch.from_numpy(ref.adjusted(host(one), **kw)).to(torch.bfloat16).cuda().repeat(times, 1)
    for other in (0, 1):
        out, obuf = rows(distinct * times, V, pad + other, "bf16", 9.0)
        L.logits_adjust("bf16", Z, out, adjust)
        L.check_device()
        assert torch.equal(out, want) and bool((obuf[:, V:] == 9.0).all())
    L.logits_adjust("bf16", Z, Z, adjust)
    assert torch.equal(Z, want) and bool((buf[:, V:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_adjust_into_rows_that_lie_between_those_of_the_logits(dtype):
    n, V = 40, 100
    for ldz, at, ldo in ((240, 112, 240), (240, 240 * 3 + 112, 240), (240, -120, 240), (720, 112, 720), (240, 240 * n - 136, 304)):
        low = -min(at, 0)
        buf = torch.full((low + max(n * ldz, max(at, 0) + n * ldo),), 7.0, device="cuda", dtype=TD[dtype])
        Z, out = buf.as_strided((n, V), (ldz, 1), low), buf.as_strided((n, V), (ldo, 1), low + at)
        Z.copy_(dev(np.random.default_rng(1).standard_normal((n, V)), dtype))
        z = host(Z)
        kw, adjust = constraints(n, V, 2)
        L.logits_adjust(dtype, Z, out, adjust)
        assert np.array_equal(host(Z), z)
        assert np.array_equal(bits(out), bits(torch.from_numpy(ref.adjusted(z, **kw)).to(TD[dtype]).cuda()))


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


@pytest.mark.parametrize("dtype,pad", [("f32", 0), ("bf16", 1)])
@pytest.mark.parametrize("n,V", [(640, 4096), (310, 16384), (2, 32001)])
@pytest.mark.parametrize("where", ["second half", "first half", "an eighth", "all but a few", "every other run"])
def test_top_of_rows_with_runs_of_nan(where, n, V, dtype, pad):
    """Whole pieces, chunks and a cluster block's share of NaN are no answers and leave the others theirs: blocks of
    128 threads, of 512, and clusters of them."""
    v = np.arange(V)
    rng = np.random.default_rng(V)
    nan = {"second half": v >= V // 2, "first half": v < V // 2, "an eighth": v * 8 // V == 2,
           "all but a few": rng.random(V) < 1 - 200 / V, "every other run": v // 512 % 2 == 0}[where]
    z = np.where(nan[None], np.nan, rng.standard_normal((n, V)) * 3)
    Z, _ = rows(n, V, pad, dtype)
    Z.copy_(dev(z, dtype))
    for K in (5, 32, 128):
        check_top(Z, K, dtype, None, host(Z).astype(np.float32))
    kw, adjust = constraints(n, V, 7)
    check_top(Z, 32, dtype, adjust, ref.adjusted(host(Z), **kw))


MANY = 609  # rows from which a block of 128 threads takes one (below, 512 threads, and clusters of blocks)


def check_top_of_repeated_rows(Z, K, dtype, adjust, adjusted, times):
    """check_top of rows that are those of `adjusted` over and over: the answer of each place is looked up."""
    n, V = Z.shape
    vals = torch.full((n, K), 5.0, device="cuda")
    ids = torch.full((n, K), 77, device="cuda", dtype=torch.int32)
    lse = torch.full((n,), 5.0, device="cuda")
    L.logits_top(dtype, Z, vals, ids, lse, adjust)
    L.check_device()
    wv, wi, wl = ref.top(adjusted, K)
    assert np.array_equal(ids.cpu().numpy(), np.tile(wi, (times, 1)))
    assert np.array_equal(vals.cpu().numpy(), np.tile(wv, (times, 1)))
    got, wl, some = host(lse), np.tile(wl, times), np.tile(np.isfinite(wl), times)
    assert np.array_equal(got[~some], wl[~some], equal_nan=True)
    if some.any():
        within(got[some], wl[some], np.tile(lse_tolerance(adjusted, V), times)[some], "lse")
    only = torch.full_like(ids, 77)
    L.logits_top(dtype, Z, vals, only, None, adjust)
    assert torch.equal(only, ids)


def repeated(kw, times):
    """`times` of the rows of an adjustment (answer_ref's names), as a LogitAdjust."""
    own = {}
    if "bias" in kw:
        own["bias"] = dev(kw["bias"])
    if "allowed" in kw:
        own["mask"] = torch.from_numpy(ref.pack_mask(kw["allowed"])).cuda()
        own["mask_row"] = ints(np.tile(kw["mask_row"], times))
    if "history" in kw:
        history = kw["history"] * times
        off = np.concatenate([[0], np.cumsum([len(h) for h in history])])
        own["history"] = ints(np.concatenate(history) if off[-1] else np.zeros(0))
        own["history_off"], own["penalty"] = ints(off, np.int64), dev(np.tile(kw["penalty"], (times, 1)))
    return L.LogitAdjust(**own)


def test_many_rows_are_as_many_as_the_library_means():
    import os
    src = open(os.path.join(os.path.dirname(L.LIB_PATH), "csrc", "top.cu")).read()
    assert f"if ((n << log_cl) <= {152} * {(MANY - 1) // 152})" in src and (MANY - 1) % 152 == 0


@pytest.mark.parametrize("dtype,pad", [("f32", 0), ("f32", 1), ("bf16", 0), ("bf16", 3)])
@pytest.mark.parametrize("K", [1, 5, 64, 128])
def test_top_of_many_rows(K, dtype, pad):
    for distinct, V in [(7, 1), (29, 31), (203, 129), (87, 2047), (29, 2048), (87, 2049), (29, 20001), (7, 49999)]:
        times = -(-MANY // distinct)
        rng = np.random.default_rng(V)
        Z, _ = rows(distinct * times, V, pad, dtype)
        one = dev(rng.standard_normal((distinct, V)) * 3, dtype)
        Z.copy_(one.repeat(times, 1))
        check_top_of_repeated_rows(Z, K, dtype, None, host(one).astype(np.float32), times)


@pytest.mark.parametrize("parts", [dict(), dict(bias=False, masks=0), dict(bias=False, history=0),
                                   dict(masks=0, history=0), dict(history=0), dict(bias=False, masks=1),
                                   dict(masks=0)])
@pytest.mark.parametrize("dtype,pad", [("f32", 0), ("f32", 2), ("bf16", 0), ("bf16", 1)])
def test_top_of_many_adjusted_rows(dtype, pad, parts):
    for distinct, V, K in [(7, 1, 2), (29, 33, 40), (203, 129, 16), (87, 8193, 128), (29, 20001, 16)]:
        times = -(-MANY // distinct)
        rng = np.random.default_rng(V)
        Z, _ = rows(distinct * times, V, pad, dtype)
        one = dev(rng.standard_normal((distinct, V)) * 3, dtype)
        Z.copy_(one.repeat(times, 1))
        kw, _ = constraints(distinct, V, V, **parts)
        check_top_of_repeated_rows(Z, K, dtype, repeated(kw, times), ref.adjusted(host(one), **kw), times)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["constant", "rising", "falling", "two values", "steps", "zeros of both signs",
                                  "one answer", "none", "not finite"])
def test_top_of_many_rows_made_to_be_hard(kind, dtype):
    """As for few rows; a block of 128 threads copies up to 128 candidates when its room is full."""
    V, v = 20003, np.arange(20003)
    z = {"constant": np.full(V, 1.5), "rising": v / 64.0, "falling": -v / 64.0,
         "two values": np.where(v % 3 == 0, 2.0, 1.0), "steps": (v // 500) * 0.5,
         "zeros of both signs": np.where(v % 2 == 0, -0.0, 0.0), "one answer": np.where(v == 12345, -3e30, -np.inf),
         "none": np.full(V, -np.inf),
         "not finite": np.where(v % 1000 == 7, np.inf, np.where(v % 1000 == 8, np.nan, -v))}[kind]
    one = dev(z[None], dtype)
    Z = one.repeat(MANY, 1)
    for K in (1, 100, 127, 128):
        check_top_of_repeated_rows(Z, K, dtype, None, host(one).astype(np.float32), MANY)


@pytest.mark.parametrize("size", [1, 128, 129, 768, 769, 1024, 1536, 1537, 3000])
def test_histories_of_every_size_of_many_rows(size):
    distinct, times, V = 29, 21, 9001
    rng = np.random.default_rng(size)
    one = dev(rng.standard_normal((distinct, V)) * 2)
    kw = dict(history=[rng.integers(0, V if i % 2 else 40, size if i % 7 else size // 2) for i in range(distinct)],
              penalty=np.stack([1 + rng.random(distinct), rng.random(distinct), rng.random(distinct) / 50],
                               1).astype(np.float32))
    want, adjust, Z = ref.adjusted(host(one), **kw), repeated(kw, times), one.repeat(times, 1)
    for K in (20, 128):
        check_top_of_repeated_rows(Z, K, "f32", adjust, want, times)
    L.logits_adjust("f32", Z, Z, adjust)
    assert np.array_equal(bits(Z), np.tile(bits(torch.from_numpy(want).cuda()), (times, 1)))


def test_one_long_history_among_short_ones():
    """The table is sized by the average: the row whose history outgrows it goes its own way."""
    distinct, times, V = 29, 21, 9001
    rng = np.random.default_rng(8)
    one = dev(rng.standard_normal((distinct, V)) * 2, "bf16")
    kw = dict(history=[rng.integers(0, V, 4000 if i == 11 else 900 if i == 20 else 30) for i in range(distinct)],
              penalty=np.tile(np.array([[1.5, -2.0, 0.1]], np.float32), (distinct, 1)))
    want = ref.adjusted(host(one), **kw)
    check_top_of_repeated_rows(one.repeat(times, 1), 33, "bf16", repeated(kw, times), want, times)


@pytest.mark.parametrize("dtype,pad", [("f32", 0), ("bf16", 1), ("bf16", 7)])
def test_many_rows_longer_than_their_bits_in_shared_memory(dtype, pad):
    distinct, times, V = 7, 88, 140001
    rng = np.random.default_rng(2)
    one = dev(rng.standard_normal((distinct, V)), dtype)
    Z, _ = rows(distinct * times, V, pad, dtype)
    Z.copy_(one.repeat(times, 1))
    kw = dict(allowed=rng.random((2, V)) < 0.9, mask_row=rng.integers(-1, 2, distinct),
              history=[np.concatenate([rng.integers(0, V, rng.integers(0, 300)), np.arange(65526, 65546)])
                       for _ in range(distinct)],
              penalty=np.tile(np.array([[0.01, -3.0, -1.0]], np.float32), (distinct, 1)))
    check_top_of_repeated_rows(Z, 33, dtype, repeated(kw, times), ref.adjusted(host(one), **kw), times)


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


@pytest.mark.parametrize("dtype,pad", [("f32", 0), ("bf16", 1), ("bf16", 7)])
@pytest.mark.parametrize("n", [1, 3, 160])
def test_rows_longer_than_their_bits_in_shared_memory(dtype, pad, n):
    """Masks and histories over several runs of 65536 elements, with tokens at the runs' ends."""
    V = 140001
    rng = np.random.default_rng(n)
    Z, _ = rows(n, V, pad, dtype)
    Z.copy_(dev(rng.standard_normal((n, V)), dtype))
    allowed = rng.random((2, V)) < 0.9
    history = [np.concatenate([rng.integers(0, V, rng.integers(0, 300)), np.arange(65526, 65546)]) for _ in range(n)]
    penalty = np.tile(np.array([[0.01, -3.0, -1.0]], np.float32), (n, 1))  # the history's tokens come first
    off = np.concatenate([[0], np.cumsum([len(h) for h in history])])
    kw = dict(allowed=allowed, mask_row=rng.integers(-1, 2, n), history=history, penalty=penalty)
    adjust = L.LogitAdjust(mask=torch.from_numpy(ref.pack_mask(allowed)).cuda(), mask_row=ints(kw["mask_row"]),
                           history=ints(np.concatenate(history)), history_off=ints(off, np.int64), penalty=dev(penalty))
    want = ref.adjusted(host(Z), **kw)
    check_top(Z, 33, dtype, adjust, want)
    out, _ = rows(n, V, 0, dtype)
    L.logits_adjust(dtype, Z, out, adjust)
    assert np.array_equal(bits(out), bits(torch.from_numpy(want).to(TD[dtype]).cuda()))


@pytest.mark.parametrize("n", [4, 400])
@pytest.mark.parametrize("size", [1, 32, 33, 512, 1023, 1024, 1025, 3000])
def test_histories_of_every_size_of_table(size, n):
    V = 9001
    rng = np.random.default_rng(size)
    z = dev(rng.standard_normal((n, V)) * 2)
    history = [rng.integers(0, V if i % 2 else 40, size) for i in range(n)]
    penalty = np.stack([1 + rng.random(n), rng.random(n), rng.random(n) / 50], 1).astype(np.float32)
    off = np.concatenate([[0], np.cumsum([len(h) for h in history])])
    adjust = L.LogitAdjust(history=ints(np.concatenate(history)), history_off=ints(off, np.int64), penalty=dev(penalty))
    want = ref.adjusted(host(z), history=history, penalty=penalty)
    check_top(z, 20, "f32", adjust, want)
    L.logits_adjust("f32", z, z, adjust)
    assert np.array_equal(bits(z), bits(torch.from_numpy(want).cuda()))


def z_bf16(z):
    return torch.from_numpy(np.asarray(z, np.float32)).to(torch.bfloat16).double().numpy()


# ------------------------------------------------------------------------------ distillation


def teacher(n, V, K, rng, share=1.0):
    """(ids, logits) of teachers' answers: K different tokens a row, some rows fewer, some none, some ids past
    the end replaced by -1, some logits -inf."""
    ids = rng.integers(0, V, (n, K)) if K > V else \
        np.argsort(rng.random((n, V)), 1)[:, :K] if n * V <= 1 << 22 else \
        (rng.integers(0, V, (n, 1)) + np.arange(K) * max(1, V // (K + 1))) % V
    logits = np.sort(rng.standard_normal((n, K)) * 3, 1)[:, ::-1].astype(np.float32)
    ids = ids.astype(np.int32)
    short = rng.random(n) < 0.2
    ids[short, K // 2 + 1:] = -1
    logits[rng.random(n) < 0.1, K - 1] = -np.inf
    out = rng.random(n) >= share
    ids[out] = -1
    return ids, logits


def distill_inputs(n, H, V, K, dtype, share=1.0, seed=0):
    rng = np.random.default_rng(seed + n + H + V + K)
    W = rng.standard_normal((V, H)) * 2.0 / np.sqrt(H)
    ids, logits = teacher(n, V, K, rng, share)
    X = rng.standard_normal((n, H)) + rng.random((n, 1)) * W[np.maximum(ids[:, 0], 0)]
    g = (0.5 + rng.random(n)).astype(np.float32) / max(n, 1)
    return dev(X, dtype), dev(W, dtype), ids, logits, g


def distill_ws(dtype, n, H, V, K):
    return torch.full((max(L.distill_workspace_bytes(dtype, n, H, V, K, op)
                           for op in (L.BG_OP_DISTILL_FWD, L.BG_OP_DISTILL_BWD)),), 0xFF, device="cuda",
                      dtype=torch.uint8)


def run_distill(dtype, X, W, ids, logits, g, tau, grad, flags=0, into=None):
    (n, K), (V, H) = ids.shape, W.shape
    t, u, gd = ints(ids), dev(logits), dev(g)
    loss, lse = (torch.full((n,), float("nan"), device="cuda") for _ in range(2))
    ws = distill_ws(dtype, n, H, V, K)
    L.distill_fwd(dtype, X, W, t, u, loss, lse, ws, tau=tau)
    dX, dW = into or (torch.full((m, H), float("nan"), device="cuda", dtype=TD[grad]) for m in (n, V))
    ws.fill_(0xFF)
    L.distill_bwd(dtype, X, W, t, u, lse, gd, grad, dX, dW, ws, tau=tau, flags=flags)
    return loss, lse, dX, dW


def distill_bounds(r, n, H, V, K, tau, grad):
    """A logit over tau: H products to 21 bits or better added in fp32 (2 u each), its division (u).  lse is as
    exact as the largest of them, to 2^-20 of itself; the loss has K terms q (log q - z) more (each to a few u,
    of at most 2 uabs + log K + zabs).  A gradient element: terms off by their probabilities' error (of P: two
    logits' errors; of Q: 4 u uabs), 2^-19 of the products' representation, and with bf16 gradients 2^-7 of P
    (its rounding in the products) and 2^-8 of the result; the sums add V u or (n + K) u of the terms'
    magnitude.  Below 2^-38 (for dW: of the largest weight) a probability may be lost."""
    dz = (2 * H * U + 2.0 ** -21) * r["zabs"]
    lse = 2 * dz + 2.0 ** -20 * (1 + np.abs(r["lse"]))
    loss = tau * tau * (lse + (K + 16) * U * (2 * r["uabs"] + 8 + r["zabs"]) + dz) + 4 * U * np.abs(r["loss"])
    term = 2 * dz + 8 * U * r["uabs"] + 2.0 ** -19 + (2.0 ** -7 if grad == "bf16" else 0)
    bX = (term + 2 * (V + K) * U) * r["absX"] + 2.0 ** -38 * r["allX"] + 2.0 ** -126
    bW = (term + 2 * (n + K) * U) * r["absW"] + 2.0 ** -38 * r["allW"] + 2.0 ** -126
    if grad == "bf16":
        bX, bW = bX + HALF * 1.01 * np.abs(r["dX"]), bW + HALF * 1.01 * np.abs(r["dW"])
    return loss, lse, bX, bW


def check_distill(dtype, grad, X, W, ids, logits, g, tau, norm=True):
    (n, K), (V, H) = ids.shape, W.shape
    got = run_distill(dtype, X, W, ids, logits, g, tau, grad)
    L.check_device()
    r = ref.distill(host(X), host(W), ids, logits, tau, g)
    if not r["rows"].any():
        assert all(not bool(t.any()) for t in got)
        return got
    loss, lse, bX, bW = distill_bounds(r, n, H, V, K, tau, grad)
    within(host(got[1]), r["lse"], lse * r["rows"], "lse")
    within(host(got[0]), r["loss"], loss * r["rows"], "loss")
    within(host(got[2]), r["dX"], bX, "dX")
    within(host(got[3]), r["dW"], bW, "dW")
    if norm and V > 1:  # roundings average out: 2^-15 of the norm in fp32, 2^-8 in bf16
        for k in ("dX", "dW"):
            off = np.linalg.norm(host(got[2 if k == "dX" else 3]) - r[k]) / np.linalg.norm(r[k])
            assert off < (2.0 ** -8 if grad == "bf16" else 2.0 ** -15), (k, off)
    return got


TYPES = [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")]


@pytest.mark.parametrize("dtype,grad", TYPES)
@pytest.mark.parametrize("n,H,V,K,tau,share", [
    (1, 32, 2, 1, 1.0, 1.0), (3, 32, 1, 2, 1.0, 1.0), (1, 128, 4001, 5, 2.0, 1.0), (2, 64, 1000, 128, 0.5, 1.0),
    (7, 96, 65, 33, 1.0, 1.0), (127, 160, 127, 2, 3.5, 0.5), (128, 256, 128, 31, 1.0, 1.0),
    (129, 192, 257, 32, 2.0, 0.7), (300, 224, 513, 64, 1.0, 0.15), (513, 256, 1023, 16, 4.0, 1.0),
    (1000, 32, 3001, 8, 1.0, 1.0), (2500, 64, 400, 100, 2.0, 0.3), (4097, 128, 130, 4, 1.0, 1.0),
    (700, 256, 2049, 12, 1.0, 0.02), (20, 64, 30, 128, 1.0, 1.0)])
def test_distill(dtype, grad, n, H, V, K, tau, share):
    X, W, ids, logits, g = distill_inputs(n, H, V, K, dtype, share)
    check_distill(dtype, grad, X, W, ids, logits, g, tau)


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_distill_of_larger_shapes(dtype, grad):
    """Several units a CTA, tiles that fall to several, entries that are sorted in several passes."""
    for n, H, V, K in ((9001, 64, 7000, 32), (3000, 256, 20001, 20), (33000, 32, 300, 8)):
        X, W, ids, logits, g = distill_inputs(n, H, V, K, dtype, 0.8)
        check_distill(dtype, grad, X, W, ids, logits, g, 2.0)


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_distill_with_one_entry_is_the_cross_entropy(dtype, grad):
    """One entry a row and tau = 1: q is one, the loss that of the token."""
    n, H, V = 700, 96, 900
    X, W, ids, logits, g = distill_inputs(n, H, V, 1, dtype, 0.8)
    got = check_distill(dtype, grad, X, W, ids, logits, g, 1.0)
    t, gd = ints(np.where(np.isinf(logits[:, 0]), -1, ids[:, 0])), dev(g)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dX, dW = (torch.empty(m, H, device="cuda", dtype=TD[grad]) for m in (n, V))
    ws = torch.empty(L.xent_workspace_bytes(dtype, n, H, V, L.BG_OP_XENT_BWD) +
                     L.xent_workspace_bytes(dtype, n, H, V, L.BG_OP_XENT_FWD), device="cuda", dtype=torch.uint8)
    L.xent_fwd(dtype, X, W, t, loss, lse, ws)
    L.xent_bwd(dtype, X, W, t, lse, gd, grad, dX, dW, ws)
    r = ref.distill(host(X), host(W), ids, logits, 1.0, g)
    b = distill_bounds(r, n, H, V, 1, 1.0, grad)
    assert torch.equal(got[1], lse)
    for a, c, tol in ((got[0], loss, b[0]), (got[2], dX, b[2]), (got[3], dW, b[3])):
        within(host(a), host(c), 2 * tol)


def test_distill_bf16_gradients_of_a_student_that_nearly_agrees():
    """Every token has an entry and the student is 2^-8 from its teacher: P rounded to bf16 alone would be as far
    off as the gradient is large; the entries' coefficients P - Q are fp32.  What is left is the result's
    rounding (2^-9 on average, 2^-8 at most), a few entries whose P rounds to the other side in the product
    (their z differs by 2^-20; 2^-11 of them, each off by 2^-7 of P: 2^-12 of the norm of P, 2^-4 of d) and the
    entries' own error, 2 dz / 2^-8."""
    n, H, V = 600, 64, 96
    rng = np.random.default_rng(2)
    W, X = dev(rng.standard_normal((V, H)) / 4, "bf16"), dev(rng.standard_normal((n, H)) / 2, "bf16")
    z = host(X) @ host(W).T
    ids = np.tile(np.arange(V, dtype=np.int32), (n, 1))
    for i in range(n):
        rng.shuffle(ids[i])
    logits = (np.take_along_axis(z, ids.astype(np.int64), 1) + 2.0 ** -8 * rng.standard_normal((n, V))).astype(np.float32)
    g = (0.5 + rng.random(n)).astype(np.float32)
    got = run_distill("bf16", X, W, ids, logits, g, 1.0, "bf16")
    r = ref.distill(host(X), host(W), ids, logits, 1.0, g)
    for k, t in (("dX", got[2]), ("dW", got[3])):
        off = np.linalg.norm(host(t) - r[k]) / np.linalg.norm(r[k])
        assert off < 2.0 ** -4, (k, off)


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_distill_of_a_token_in_several_entries(dtype, grad):
    n, H, V, K = 200, 64, 300, 40
    X, W, ids, logits, g = distill_inputs(n, H, V, K, dtype)
    rng = np.random.default_rng(1)
    ids[:100] = np.where(ids[:100] >= 0, rng.integers(0, 3, (100, K)), -1)
    ids[100:110] = np.where(ids[100:110] >= 0, 7, -1)
    check_distill(dtype, grad, X, W, ids, logits, g, 1.5)


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_distill_rows_left_out_may_hold_anything(dtype, grad):
    """Rows without an entry, or with entries of -inf alone: their X, g and lse are not used."""
    n, H, V, K = 300, 64, 200, 6
    X, W, ids, logits, g = distill_inputs(n, H, V, K, dtype, 0.5)
    logits[5:9] = -np.inf
    r = ref.distill(host(X), host(W), ids, logits, 2.0, g)
    out = torch.from_numpy(~r["rows"]).cuda()
    want = run_distill(dtype, X, W, ids, logits, g, 2.0, grad)
    X[out] = float("nan")
    g = np.where(r["rows"], g, np.nan).astype(np.float32)
    logits = np.where(ids < 0, np.nan, logits).astype(np.float32)
    got = run_distill(dtype, X, W, ids, logits, g, 2.0, grad)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for a in (got[0], got[1], got[2]):
        assert not bool(a[out].any())


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_distill_of_entries_of_the_lowest_value(dtype, grad):
    """Beside larger entries the lowest value has q = 0, as an entry that is none; a row of nothing else is one of
    equal logits.  At tau < 1 their quotients by tau pass the type's range."""
    n, H, V, K, tau = 300, 64, 200, 6, 0.5
    X, W, ids, logits, g = distill_inputs(n, H, V, K, dtype)
    rng = np.random.default_rng(4)
    low = rng.random((n, K)) < 0.4
    low[:, 0] &= ids[:, 1] < 0
    low[50:60] = True
    logits[50:60] = np.where(np.isinf(logits[50:60]), -np.inf, 0.0)
    mixed = ((ids >= 0) & ~np.isinf(logits) & ~low).any(1)
    same = np.where(low & mixed[:, None], -1, ids).astype(np.int32)
    equal = np.where(low & ~mixed[:, None] & ~np.isinf(logits), 0.0, logits).astype(np.float32)
    lowest = np.where(low & ~np.isinf(logits), np.finfo(np.float32).min, logits).astype(np.float32)
    r = ref.distill(host(X), host(W), same, equal, tau, g)
    assert r["rows"][50:60].any() and (low & mixed[:, None] & (ids >= 0)).any()
    for a, k, tol in zip(run_distill(dtype, X, W, ids, lowest, g, tau, grad), ("loss", "lse", "dX", "dW"),
                         distill_bounds(r, n, H, V, K, tau, grad)):
        within(host(a), r[k], tol)


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_distill_with_no_row_left(dtype, grad):
    X, W, ids, logits, g = distill_inputs(150, 64, 300, 5, dtype, 0.0)
    ids[:] = -1
    check_distill(dtype, grad, X, W, ids, logits, g, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_accumulates_and_skips_what_is_not_asked(dtype):
    n, H, V, K = 400, 96, 500, 9
    X, W, ids, logits, g = distill_inputs(n, H, V, K, dtype, 0.7)
    rng = np.random.default_rng(0)
    old = [rng.standard_normal((m, H)).astype(np.float32) for m in (n, V)]
    r = ref.distill(host(X), host(W), ids, logits, 2.0, g)
    _, _, bX, bW = distill_bounds(r, n, H, V, K, 2.0, "f32")
    _, lse, dX, dW = run_distill(dtype, X, W, ids, logits, g, 2.0, "f32", flags=L.BG_ACCUM,
                                 into=[dev(o) for o in old])
    # two additions to what was there
    within(host(dX), old[0] + r["dX"], bX + 3 * U * (np.abs(old[0]) + r["absX"]))
    within(host(dW), old[1] + r["dW"], bW + 3 * U * (np.abs(old[1]) + r["absW"]))
    for grad in ("f32", "bf16") if dtype == "bf16" else ("f32",):
        _, _, wX, wW = run_distill(dtype, X, W, ids, logits, g, 2.0, grad)
        t, u, gd, ws = ints(ids), dev(logits), dev(g), distill_ws(dtype, n, H, V, K)
        for which in (0, 1):
            into = [torch.full((m, H), float("nan"), device="cuda", dtype=TD[grad]) if k == which else None
                    for k, m in enumerate((n, V))]
            ws.fill_(0xFF)
            L.distill_bwd(dtype, X, W, t, u, lse, gd, grad, into[0], into[1], ws, tau=2.0)
            want = (wX, wW)[which]
            # (alone it has all CTAs: sums in another order)
            within(host(into[which]), host(want), (bX, bW)[which] + 2 * HALF * np.abs(host(want)) * (grad == "bf16"))


def test_distill_reports_tokens_past_the_vocabulary():
    n, H, V, K = 90, 64, 100, 4
    X, W, ids, logits, g = distill_inputs(n, H, V, K, "bf16")
    bad = ids.copy()
    bad[3, 1], bad[40] = V, V + 7
    r = ref.distill(host(X), host(W), bad, logits, 1.0, g)
    got = run_distill("bf16", X, W, bad, logits, g, 1.0, "f32")
    with pytest.raises(L.BandGGNNError, match="site 135"):
        L.check_device()
    loss, _, bX, _ = distill_bounds(r, n, H, V, K, 1.0, "f32")
    within(host(got[0]), r["loss"], loss * r["rows"])
    within(host(got[2]), r["dX"], bX)
    L.check_device()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tau", [1.0, 3.0])
def test_distill_gradient_against_differences(dtype, tau):
    """Directional differences of the forward itself.  With step e along a direction whose logits (over tau) move
    by at most m, the central difference is off by e^2 m^3 / 6 of the weights' sum times tau^2, and by the loss's
    rounding over e."""
    n, H, V, K = 96, 64, 200, 12
    X, W, ids, logits, g = distill_inputs(n, H, V, K, dtype)
    rng = np.random.default_rng(3)
    r = ref.distill(host(X), host(W), ids, logits, tau, g)
    _, _, dX, dW = run_distill(dtype, X, W, ids, logits, g, tau, "f32")
    Xf, Wf = X.float(), W.float()
    for which, d in (("X", dX), ("W", dW)):
        Dd = dev(rng.standard_normal(tuple(d.shape)))
        move = host(Dd) @ host(Wf).T if which == "X" else host(Xf) @ host(Dd).T
        m = 2 * np.abs(move).max() / tau
        e = 0.02 / m
        f = []
        for s in (e, -e):
            args = (Xf + s * Dd, Wf) if which == "X" else (Xf, Wf + s * Dd)
            f.append(float((host(run_distill("f32", *args, ids, logits, g, tau, "f32")[0]) * g).sum()))
        got, want = float((host(d) * host(Dd)).sum()), (f[0] - f[1]) / (2 * e)
        loss, _, _, _ = distill_bounds(r, n, H, V, K, tau, "f32")
        # X + e D itself is rounded to fp32: a logit moves by u of its magnitude
        tol = g.sum() * (tau * tau * (e * m) ** 2 * m / 6 + (loss.max() + 2 * tau * tau * U * r["zabs"]) / e)
        assert abs(got - want) <= tol, (which, got, want, tol)


@pytest.mark.parametrize("dtype,grad", TYPES)
def test_distill_gives_the_same_bits_again(dtype, grad):
    X, W, ids, logits, g = distill_inputs(3000, 64, 900, 24, dtype, 0.8)
    first = run_distill(dtype, X, W, ids, logits, g, 2.0, grad)
    for _ in range(3):
        for a, b in zip(run_distill(dtype, X, W, ids, logits, g, 2.0, grad), first):
            assert torch.equal(a, b)


def test_distill_of_enormous_logits_stays_within_its_rows():
    """Rows with |lse| beyond 2^20 have gradients of no meaning, but finite ones; the other rows keep theirs."""
    n, H, V, K = 200, 64, 150, 8
    for grad in ("f32", "bf16"):
        X, W, ids, logits, g = distill_inputs(n, H, V, K, "bf16")
        want = run_distill("bf16", X, W, ids, logits, g, 1.0, grad)
        X[::20] *= 1e9
        got = run_distill("bf16", X, W, ids, logits, g, 1.0, grad)
        keep = torch.ones(n, dtype=torch.bool)
        keep[::20] = False
        r = ref.distill(host(X)[keep], host(W), ids[keep.numpy()], logits[keep.numpy()], 1.0, g[keep.numpy()])
        _, _, bX, _ = distill_bounds(r, n, H, V, K, 1.0, grad)
        within(host(got[2])[keep.numpy()], host(want[2])[keep.numpy()], 2 * bX)
        assert all(bool(torch.isfinite(t).all()) for t in got)


# ------------------------------------------------------------------------------ all of them together


def answer_and_learn(teacher_x, teacher_w, x, w, adjust, bufs, stream=None):
    """A teacher's answers under a grammar, and the student's loss and gradients on them."""
    Z, u, t, tlse, loss, lse, g, dX, dW, ws = bufs
    L.logits_fwd("bf16", teacher_x, teacher_w, "bf16", Z, stream=stream)
    L.logits_top("bf16", Z, u, t, tlse, adjust, stream=stream)
    L.logits_adjust("bf16", Z, Z, adjust, stream=stream)
    L.distill_fwd("bf16", x, w, t, u, loss, lse, ws, tau=2.0, stream=stream)
    L.distill_bwd("bf16", x, w, t, u, lse, g, "f32", dX, dW, ws, tau=2.0, stream=stream)


def test_a_student_learns_from_a_teachers_answers_on_its_stream_and_in_a_graph():
    """The operators one after the other, as they are used: on a side stream, and captured and replayed on new
    values (with an adjustment that changes between replays)."""
    n, H, V, K = 600, 64, 777, 16
    rng = np.random.default_rng(9)
    tx, tw = dev(rng.standard_normal((n, H)), "bf16"), dev(rng.standard_normal((V, H)) / 4, "bf16")
    x, w = dev(rng.standard_normal((n, H)), "bf16"), dev(rng.standard_normal((V, H)) / 4, "bf16")
    kw, adjust = constraints(n, V, 5)
    g = rng.random(n).astype(np.float32)

    def make():
        Z, _ = rows(n, V, 3, "bf16", 0.0)
        return [Z, torch.zeros(n, K, device="cuda"), torch.zeros(n, K, device="cuda", dtype=torch.int32),
                torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), dev(g),
                torch.zeros(n, H, device="cuda"), torch.zeros(V, H, device="cuda"), distill_ws("bf16", n, H, V, K)]

    bufs = make()
    st = torch.cuda.Stream()
    x2 = torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        x2.copy_(x)
    answer_and_learn(tx, tw, x2, w, adjust, bufs, stream=st)
    st.synchronize()
    L.check_device()
    z = torch.empty(n, V, device="cuda", dtype=torch.bfloat16)
    L.logits_fwd("bf16", tx, tw, "bf16", z)
    adj = ref.adjusted(host(z), **kw)
    vals, ids, _ = ref.top(adj, K)
    assert np.array_equal(bits(bufs[0]), bits(torch.from_numpy(adj).to(torch.bfloat16).cuda()))
    assert np.array_equal(bufs[2].cpu().numpy(), ids) and np.array_equal(bufs[1].cpu().numpy(), vals)
    r = ref.distill(host(x), host(w), ids, vals, 2.0, g)
    loss, lse, bX, bW = distill_bounds(r, n, H, V, K, 2.0, "f32")
    within(host(bufs[4]), r["loss"], loss * r["rows"])
    within(host(bufs[7]), r["dX"], bX)
    within(host(bufs[8]), r["dW"], bW)
    again = make()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        answer_and_learn(tx, tw, x2, w, adjust, again)
    adjust._kept["bias"].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(again[2], bufs[2])
    adjust._kept["bias"].copy_(dev(kw["bias"]))
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(again[:9], bufs[:9]):
        assert np.array_equal(bits(a), bits(b)) if a.dtype != torch.int32 else torch.equal(a, b)


def test_graphs_that_share_a_workspace_replay_one_after_the_other():
    """Two captured training steps over one workspace, replayed in turn: nothing in it outlives a call."""
    n, H, V, K = 500, 64, 700, 10
    steps = []
    ws = distill_ws("bf16", n, H, V, K)
    for seed in (1, 2):
        X, W, ids, logits, g = distill_inputs(n, H, V, K, "bf16", 0.8, seed)
        want = run_distill("bf16", X, W, ids, logits, g, 2.0, "f32")
        outs = [torch.zeros_like(t) for t in want]
        args = (ints(ids), dev(logits))
        gd = dev(g)

        def step(X=X, W=W, args=args, gd=gd, outs=outs):
            L.distill_fwd("bf16", X, W, *args, outs[0], outs[1], ws, tau=2.0)
            L.distill_bwd("bf16", X, W, *args, outs[1], gd, "f32", outs[2], outs[3], ws, tau=2.0)

        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        steps.append((graph, outs, want, step))  # (step: what the graph reads stays where it is)
    for k in (0, 1, 1, 0, 1, 0):
        for t in steps[k][1]:
            t.zero_()
        steps[k][0].replay()
        torch.cuda.synchronize()
        for a, b in zip(steps[k][1], steps[k][2]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_top_and_adjust_give_the_same_bits_again(dtype):
    """Blocks raise their bounds as they find each other's: what is done differs from run to run, its result does
    not (lse included: each thread's sum, and the order in which they are joined, are fixed)."""
    n, V, K = 700, 20001, 40
    rng = np.random.default_rng(11)
    z = dev(np.round(rng.standard_normal((n, V)) * 8) / 4, dtype)  # ties
    kw, adjust = constraints(n, V, 3)
    first = None
    for _ in range(6):
        got = [torch.empty(n, K, device="cuda"), torch.empty(n, K, device="cuda", dtype=torch.int32)]
        L.logits_top(dtype, z, got[0], got[1], None, adjust)
        out = torch.empty_like(z)
        L.logits_adjust(dtype, z, out, adjust)
        got.append(torch.nan_to_num(out, nan=1.0))
        if first is None:
            first = got
        for a, b in zip(got, first):
            assert torch.equal(a, b)
    assert np.array_equal(first[1].cpu().numpy(), ref.top(ref.adjusted(host(z), **kw), K)[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [2, 300, 700])
def test_lse_of_rows_with_dense_histories_has_the_same_bits_again(n, dtype):
    """Tables half full and more, whose tokens make most of the sum: the order in which their exponentials are added
    is that of the tokens' places, which must not depend on which thread came first."""
    V, K = 20001, 5
    rng = np.random.default_rng(n)
    z = dev(rng.standard_normal((n, V)), dtype)
    history = [rng.integers(0, V, m) for m in rng.integers(900, 1500, n)]
    penalty = np.tile(np.array([[0.5, -6.0, -0.5]], np.float32), (n, 1))
    off = np.concatenate([[0], np.cumsum([len(h) for h in history])])
    adjust = L.LogitAdjust(history=ints(np.concatenate(history)), history_off=ints(off, np.int64), penalty=dev(penalty))
    check_top(z, K, dtype, adjust, ref.adjusted(host(z), history=history, penalty=penalty))
    vals, ids = torch.empty(n, K, device="cuda"), torch.empty(n, K, device="cuda", dtype=torch.int32)
    first = None
    for _ in range(20):
        lse = torch.full((n,), float("nan"), device="cuda")
        L.logits_top(dtype, z, vals, ids, lse, adjust)
        first = lse if first is None else first
        assert torch.equal(lse, first)


FIRST_CALLS = """
import torch
from paper_1906_11786_gb300 import lib as L
n, H, V, K = 500, 64, 300, 8
gen = torch.Generator(device="cuda").manual_seed(1)
X, W = (torch.randn(m, H, device="cuda", generator=gen) for m in (n, V))
g, bias = torch.ones(n, device="cuda"), torch.randn(V, device="cuda", generator=gen)
ws = torch.empty(max([L.logits_workspace_bytes("f32", n, H, V)] +
                     [L.distill_workspace_bytes("f32", n, H, V, K, op)
                      for op in (L.BG_OP_DISTILL_FWD, L.BG_OP_DISTILL_BWD)]), device="cuda", dtype=torch.uint8)
outs = [torch.zeros(*s, device="cuda") for s in ((n, V), (n, V), (n, K), (n,), (n,), (n, H), (V, H))]
Z, Y, u, loss, lse, dX, dW = outs
t = torch.zeros(n, K, device="cuda", dtype=torch.int32)
adjust = L.LogitAdjust(bias=bias)

def calls():
    L.logits_fwd("f32", X, W, "f32", Z, ws)
    L.logits_adjust("f32", Z, Y, adjust)
    L.logits_top("f32", Z, u, t, None, adjust)
    L.distill_fwd("f32", X, W, t, u, loss, lse, ws)
    L.distill_bwd("f32", X, W, t, u, lse, g, "f32", dX, dW, ws)

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


def test_the_first_calls_of_a_process_can_be_captured():
    import os
    import subprocess
    import sys
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, timeout=300,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]
