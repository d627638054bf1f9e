"""The operators that answer with a vocabulary without a GPU: refusals, sizes, the binding's checks."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest

import answer_ref as ref
from paper_1906_11786_gb300 import _binding as L
from paper_1906_11786_gb300 import build as B

A = 1 << 20  # an aligned address that is never read
BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return L.load()


def _refused(rc, word, code=-1):
    assert rc == code, rc
    assert word in L.load().bg_last_error().decode()


def _adjust(**kw):
    return ctypes.byref(L.bg_adjust(**kw))


def test_binding_struct_matches_the_c_layout(tmp_path):
    """bg_adjust has the header's fields in its order, at the offsets and size that the C compiler gives them."""
    import re
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    src = re.sub(r"/\*.*?\*/", "", open(L.HEADER).read(), flags=re.S)
    fields = re.findall(r"(\w+)\s*;", re.search(r"struct bg_adjust \{(.*?)\};", src, flags=re.S).group(1))
    assert [f for f, _ in L.bg_adjust._fields_] == fields
    prog = "#include <stdio.h>\n#include <stddef.h>\n#include \"bandggnn.h\"\nint main(void) {\n" + "".join(
        f'  printf("%zu\\n", offsetof(bg_adjust, {f}));\n' for f in fields) + \
        '  printf("%zu\\n", sizeof(bg_adjust));\n  return 0;\n}\n'
    (tmp_path / "a.c").write_text(prog)
    import os
    subprocess.run([cc, "-I", os.path.dirname(L.HEADER), str(tmp_path / "a.c"), "-o", str(tmp_path / "a")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "a")], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [getattr(L.bg_adjust, f).offset for f in fields] + [ctypes.sizeof(L.bg_adjust)]


def test_reference_masks_number_bits_as_stated():
    allowed = np.random.default_rng(0).random((3, 77)) < 0.5
    words = ref.pack_mask(allowed).view(np.uint32)
    assert words.shape == (3, 3)
    for v in range(77):
        assert np.array_equal((words[:, v // 32] >> np.uint32(v % 32)) & 1, allowed[:, v])


@pytest.mark.parametrize("n,H,V,word", [(-1, 64, 9, "n must"), ((1 << 29) + 1, 64, 9, "n must"),
                                        (8, 48, 9, "H must"), (8, 288, 9, "H must"), (8, 64, 0, "V must"),
                                        (8, 64, (1 << 24) + 1, "V must")])
def test_shapes_out_of_range_are_refused(lib, n, H, V, word):
    ld = max(V, 1)
    _refused(lib.bg_logits_fwd(L.BG_F32, n, H, V, A, A, L.BG_F32, ld, A, A, BIG, None), word)
    assert lib.bg_logits_workspace_bytes(L.BG_F32, n, H, V) == 0
    if word != "H must":
        _refused(lib.bg_logits_adjust(L.BG_F32, n, V, ld, A, None, ld, A, None), word)
        _refused(lib.bg_logits_top(L.BG_F32, n, V, ld, A, None, 4, A, A, A, None), word)


def test_pointers_types_and_strides_are_checked(lib):
    odd = A + 8
    f = L.BG_F32
    _refused(lib.bg_logits_fwd(7, 8, 64, 9, A, A, f, 9, A, A, BIG, None), "dtype")
    _refused(lib.bg_logits_fwd(f, 8, 64, 9, A, A, 7, 9, A, A, BIG, None), "dtype")
    _refused(lib.bg_logits_fwd(f, 8, 64, 9, A, A, f, 8, A, A, BIG, None), "ldz must")
    _refused(lib.bg_logits_fwd(f, 8, 64, 9, A, A, f, (1 << 31) + 1, A, A, BIG, None), "ldz must")
    _refused(lib.bg_logits_fwd(f, 8, 64, 9, None, A, f, 9, A, A, BIG, None), "X is NULL")
    _refused(lib.bg_logits_fwd(f, 8, 64, 9, A, odd, f, 9, A, A, BIG, None), "W not 16-byte")
    _refused(lib.bg_logits_fwd(f, 8, 64, 9, A, A, f, 9, odd, A, BIG, None), "Z not 16-byte")
    need = lib.bg_logits_workspace_bytes(f, 5, 64, 9)
    assert need > 0 == lib.bg_logits_workspace_bytes(f, 4, 64, 9)
    assert lib.bg_logits_workspace_bytes(L.BG_BF16, 800, 64, 9) == 0
    _refused(lib.bg_logits_fwd(f, 5, 64, 9, A, A, f, 9, A, A, need - 1, None), "workspace", code=-2)
    _refused(lib.bg_logits_fwd(f, 5, 64, 9, A, A, f, 9, A, None, BIG, None), "ws is NULL")
    _refused(lib.bg_logits_adjust(5, 8, 9, 9, A, None, 9, A, None), "dtype")
    _refused(lib.bg_logits_adjust(f, 8, 9, 9, A, None, 8, A, None), "ldo must")
    _refused(lib.bg_logits_adjust(f, 8, 9, 9, A, None, 10, A, None), "in place")
    _refused(lib.bg_logits_adjust(f, 8, 9, 9, odd, None, 9, A, None), "Z not 16-byte")
    for K in (0, -1, 129):
        _refused(lib.bg_logits_top(f, 8, 9, 9, A, None, K, A, A, A, None), "K must")
    _refused(lib.bg_logits_top(f, 8, 9, 9, A, None, 2, None, A, A, None), "top_logit is NULL")
    _refused(lib.bg_logits_top(f, 8, 9, 9, A, None, 2, A, A, odd, None), "lse not 16-byte")


def test_results_over_other_rows_of_the_logits_are_refused(lib):
    """out is Z or has no element in common with it, whatever the distances between rows."""
    def adjust(dt, n, V, ldz, out, ldo):
        return lib.bg_logits_adjust(dt, n, V, ldz, A, None, ldo, out, None)

    f, b = L.BG_F32, L.BG_BF16
    for dt, e in ((f, 4), (b, 2)):
        step = 16 // e  # elements of 16 bytes
        for n, V, ldz, at, ldo in [(1, 100, 100, step, 100), (1, 100, 100, -step, 100), (8, 100, 104, 104, 104),
                                   (8, 100, 104, -104, 104), (8, 100, 240, 96, 240), (8, 100, 240, 240 * 7 - 96, 240),
                                   (8, 100, 240, 240 + 96, 240), (8, 100, 240, -96, 240), (8, 100, 200, 104, 208),
                                   (8, 100, 104, -8 * 200 + 104, 200), (1 << 20, 8, 16, 8, 24), (3, 100, 100, 296, 1000)]:
            _refused(adjust(dt, n, V, ldz, A + at * e, ldo), "out overlaps Z")


@pytest.mark.parametrize("kw,word", [
    (dict(bias=A + 4), "bias not 16-byte"), (dict(mask=A), "n_masks must be 1"),
    (dict(mask=A, n_masks=-2), "n_masks must be 1"), (dict(mask=A, n_masks=7), "at least n"),
    (dict(mask_row=A), "without adjust.mask"), (dict(n_masks=2), "without adjust.mask"),
    (dict(history=A, history_len=-1, history_off=A, penalty=A), "history_len < 0"),
    (dict(history=A, history_len=1, history_off=A), "belong together"), (dict(penalty=A), "belong together"),
    (dict(history_len=3, history_off=A, penalty=A), "without adjust.history"),
    (dict(history=A, history_len=3), "without adjust.history"),
    (dict(history=A, history_len=1, history_off=A, penalty=A + 4), "penalty not 16-byte")])
def test_adjustments_are_checked(lib, kw, word):
    adjust = _adjust(**kw)
    _refused(lib.bg_logits_adjust(L.BG_F32, 8, 9, 9, A, adjust, 9, A, None), word)
    _refused(lib.bg_logits_top(L.BG_BF16, 8, 9, 9, A, adjust, 2, A, A, A, None), word)


def test_distillation_checks_its_arguments(lib):
    f, b = L.BG_F32, L.BG_BF16

    def fwd(dt=f, n=8, H=64, V=9, K=4, X=A, W=A, ids=A, u=A, tau=1.0, loss=A, lse=A, ws=A, size=BIG):
        return lib.bg_distill_fwd(dt, n, H, V, K, X, W, ids, u, tau, loss, lse, ws, size, None)

    def bwd(dt=f, n=8, H=64, V=9, K=4, X=A, W=A, ids=A, u=A, tau=1.0, lse=A, g=A, gd=f, dX=A, dW=A, flags=0, ws=A,
            size=BIG):
        return lib.bg_distill_bwd(dt, n, H, V, K, X, W, ids, u, tau, lse, g, gd, dX, dW, flags, ws, size, None)

    for call in (fwd, bwd):
        for kw, word in ((dict(dt=9), "dtype"), (dict(n=-1), "n must"), (dict(H=48), "H must"), (dict(V=0), "V must"),
                         (dict(K=0), "K must"), (dict(K=129), "K must"), (dict(n=1 << 29, K=2), "n K must"),
                         (dict(tau=0.0), "tau must"), (dict(tau=-1.0), "tau must"), (dict(tau=1e4), "tau must"),
                         (dict(tau=float("nan")), "tau must"), (dict(W=None), "W is NULL"), (dict(X=A + 8), "X not"),
                         (dict(ids=None), "top_id is NULL"), (dict(u=A + 4), "top_logit not"),
                         (dict(ws=None), "ws is NULL"), (dict(lse=None), "lse is NULL")):
            _refused(call(**kw), word)
    for dt in (f, b):
        for op, call in ((L.BG_OP_DISTILL_FWD, fwd), (L.BG_OP_DISTILL_BWD, bwd)):
            need = lib.bg_distill_workspace_bytes(dt, 8, 64, 9, 4, op)
            assert need > 0
            _refused(call(dt=dt, size=need - 1), "workspace", code=-2)
    _refused(fwd(loss=None), "loss is NULL")
    _refused(bwd(g=None), "dloss is NULL")
    _refused(bwd(gd=b), "fp32 gradients")
    _refused(bwd(dt=b, gd=b, flags=1), "BG_ACCUM")
    _refused(bwd(flags=2), "flags")
    _refused(bwd(dX=None, dW=None), "dX and dW")
    _refused(bwd(gd=4), "dtype")
    for bad in ((f, -1, 64, 9, 4, 7), (f, 8, 40, 9, 4, 7), (f, 8, 64, 9, 0, 7), (f, 8, 64, 9, 4, L.BG_OP_XENT_FWD),
                (5, 8, 64, 9, 4, 7), (f, 1 << 29, 64, 9, 2, 7)):
        assert lib.bg_distill_workspace_bytes(*bad) == 0


def test_distillation_workspaces_do_not_hold_the_logits(lib):
    n, H, V, K = 1 << 20, 256, 1 << 20, 64
    for dt in (L.BG_F32, L.BG_BF16):
        for op in (L.BG_OP_DISTILL_FWD, L.BG_OP_DISTILL_BWD):
            assert 0 < lib.bg_distill_workspace_bytes(dt, n, H, V, K, op) < 64 * H * (n + V) + 24 * n * K * (1 + H // 32)


def test_nothing_to_do_is_done_without_a_device(lib):
    f, b = L.BG_F32, L.BG_BF16
    assert lib.bg_distill_fwd(f, 0, 64, 9, 4, None, A, None, None, 1.0, None, None, None, 0, None) == 0
    for grad in (f, b):
        assert lib.bg_distill_bwd(b, 0, 64, 9, 4, None, A, None, None, 1.0, None, None, grad, None, None, 0, None, 0,
                                  None) == 0
    assert lib.bg_distill_bwd(f, 0, 64, 9, 4, None, A, None, None, 1.0, None, None, f, None, A, L.BG_ACCUM, None, 0,
                              None) == 0
    assert lib.bg_logits_fwd(L.BG_F32, 0, 64, 9, None, A, L.BG_F32, 9, None, None, 0, None) == 0
    assert lib.bg_logits_adjust(L.BG_BF16, 0, 9, 9, None, None, 9, None, None) == 0
    assert lib.bg_logits_top(L.BG_BF16, 0, 9, 9, None, None, 3, None, None, None, None) == 0


def test_workspaces_grow_with_the_operands_alone(lib):
    for n, H, V in ((5, 32, 1), (1 << 20, 256, 1 << 20)):
        need = lib.bg_logits_workspace_bytes(L.BG_F32, n, H, V)
        assert 0 < need < 6 * H * (n + V + 512) + 4096


def test_sums_by_token_are_cut_for_as_many_blocks_as_an_sm_holds(lib):
    """228 KB of shared memory an SM, of which each block takes 1 KB beside its own (256 bytes of them fixed)."""
    resident = lib["_ZN2bg18token_sum_residentEliiPi"]
    resident.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
    smem = ctypes.c_int()
    for weighted in (0, 1):
        for H in range(32, 257, 32):
            for n in [1, 100, 10 ** 4, 311296, 311297, 450000, 466944, 466945, 933888, 1300000, 1 << 21, 1 << 29]:
                blocks = resident(n, H, weighted, ctypes.byref(smem))
                assert blocks >= 2 and blocks * (smem.value + 256 + 1024) <= 228 * 1024, (n, H, weighted)


class _Elsewhere:
    """What the binding reads of a CUDA tensor, on a device of choice."""

    def __init__(self, device, dtype, *shape, strides=None):
        self.device_index, self.dtype, self.shape, self.is_cuda = device, dtype, shape, True
        self.strides = strides

    def numel(self):
        n = 1
        for m in self.shape:
            n *= m
        return n

    def stride(self, i):
        return self.strides[i] if self.strides else (self.shape[1] if i == 0 else 1)

    def dim(self):
        return len(self.shape)

    element_size = data_ptr = lambda self: A
    is_contiguous = lambda self: True
    get_device = lambda self: self.device_index


def test_tensors_of_another_device_are_refused(monkeypatch):
    import torch
    monkeypatch.setattr(L, "_current_device", lambda: 0)
    f, i = torch.float32, torch.int32
    n, V, H, K = 6, 9, 64, 3
    args = {"X": (f, n, H), "W": (f, V, H), "Z": (f, n, V), "out": (f, n, V), "ws": (f, 1 << 20),
            "top_logit": (f, n, K), "top_id": (i, n, K), "lse": (f, n), "loss": (f, n), "dloss": (f, n),
            "dX": (f, n, H), "dW": (f, V, H)}
    calls = [("X W Z ws", lambda X, W, Z, ws: L.logits_fwd("f32", X, W, "f32", Z, ws)),
             ("Z out", lambda Z, out: L.logits_adjust("f32", Z, out, None)),
             ("Z top_logit top_id lse", lambda *t: L.logits_top("f32", *t)),
             ("X W top_id top_logit loss lse ws", lambda *t: L.distill_fwd("f32", *t)),
             ("X W top_id top_logit lse dloss dX dW ws", lambda *t: L.distill_bwd("f32", *t[:6], "f32", *t[6:]))]
    for names, call in calls:
        for away in names.split():
            with pytest.raises(ValueError, match=f"^{away} is on cuda:1, the current device is cuda:0"):
                call(*(_Elsewhere(int(name == away), *args[name]) for name in names.split()))
    there = L.LogitAdjust(bias=_Elsewhere(1, f, V))
    with pytest.raises(ValueError, match="adjust is on cuda:1"):
        L.logits_adjust("f32", _Elsewhere(0, f, n, V), _Elsewhere(0, f, n, V), there)
    with pytest.raises(ValueError, match="on one device"):
        L.LogitAdjust(bias=_Elsewhere(1, f, V), mask=_Elsewhere(0, i, 1, 1))


def test_binding_checks_types_shapes_and_strides(monkeypatch):
    import torch
    monkeypatch.setattr(L, "_current_device", lambda: 0)
    f, i, q = torch.float32, torch.int32, torch.int64
    n, V = 6, 40
    Z = _Elsewhere(0, f, n, V)
    for strides in ((V - 1, 1), (2 * V, 2), (1, n)):
        with pytest.raises(ValueError, match="Z must have rows"):
            L.logits_top("f32", _Elsewhere(0, f, n, V, strides=strides), Z, Z)
    with pytest.raises(ValueError, match="CUDA tensor"):
        L.logits_adjust("f32", torch.zeros(n, V), torch.zeros(n, V), None)
    with pytest.raises(ValueError, match="Z must be torch.bfloat16"):
        L.logits_adjust("bf16", Z, Z, None)
    with pytest.raises(ValueError, match="belong together"):
        L.LogitAdjust(history=_Elsewhere(0, i, 3))
    with pytest.raises(ValueError, match="without a mask"):
        L.LogitAdjust(mask_row=_Elsewhere(0, i, n))
    with pytest.raises(ValueError, match="bias must be torch.float32"):
        L.LogitAdjust(bias=_Elsewhere(0, i, V))
    with pytest.raises(ValueError, match="history_off must be torch.int64"):
        L.LogitAdjust(history=_Elsewhere(0, i, 3), history_off=_Elsewhere(0, i, n + 1), penalty=_Elsewhere(0, f, n, 3))
    ok = dict(history=_Elsewhere(0, i, 3), history_off=_Elsewhere(0, q, n + 1), penalty=_Elsewhere(0, f, n, 3))
    for kw, word in ((dict(bias=_Elsewhere(0, f, V + 1)), "bias must be"),
                     (dict(mask=_Elsewhere(0, i, 1, 1)), "mask must be"),
                     (dict(mask=_Elsewhere(0, i, 1, 2), mask_row=_Elsewhere(0, i, n + 1)), "mask_row must be"),
                     (dict(ok, penalty=_Elsewhere(0, f, n, 2)), "penalty must be"),
                     (dict(ok, history_off=_Elsewhere(0, q, n)), "history_off must be")):
        with pytest.raises(ValueError, match=word):
            L.logits_adjust("f32", Z, Z, L.LogitAdjust(**kw))


def test_every_barrier_of_the_logits_kernel_is_initialised():
    import os
    import re
    src = open(os.path.join(os.path.dirname(L.LIB_PATH), "csrc", "logits.cu")).read()
    fields = {f.split("[")[0].strip()
              for f in re.search(r"struct Bars \{\s*uint64_t ([^;]*);", src).group(1).split(",")}
    init = set(re.findall(r"mbar_init\(&bars->(\w+)", src))
    used = set(re.findall(r"&bars->(\w+)", src)) - {"tmem", "abort"}
    assert init == fields == used, (fields, init, used)
