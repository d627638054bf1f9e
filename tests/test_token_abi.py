"""Token operators without a GPU: the generator's published test vectors, refusals, sizes."""
from __future__ import annotations

import pytest
import token_ref as ref

from paper_1906_11786_gb300 import _binding as L
from paper_1906_11786_gb300 import build as B

LOW = ref.LOW
P16 = 1 << 20  # an aligned address that is never read


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return L.load()


def test_reference_generator_matches_the_published_vectors():
    """The known answers that Random123 (Salmon et al.) gives for 7 rounds."""
    want = {(0, 0): "5f6fb709 0d893f64 4f121f81 4f730a48",
            (LOW, LOW): "5207ddc2 45165e59 4d8ee751 8c52f662"}
    for (c, k), words in want.items():
        got = ref.philox_scalar([c] * 4, [k] * 2)
        assert " ".join(f"{w:08x}" for w in got) == words


def test_reference_mask_numbers_elements_as_stated():
    seed, call, p = 0x0123456789ABCDEF, 0x7EDCBA9876543210, 0.375
    got = ref.keep(3, 50, p, seed, call)
    for j in range(50):
        i = 3 + j
        w = ref.philox_scalar([i // 8 & LOW, i // 8 >> 32, call & LOW, call >> 32],
                              [seed & LOW, seed >> 32])
        bits = (w[(i % 8) // 2] >> (16 * (i % 2))) & 0xFFFF
        assert got[j] == (bits >= 24576)


def _refused(rc, word, code=-1):
    assert rc == code, rc
    assert word in L.load().bg_last_error().decode()


@pytest.mark.parametrize("p", [-0.1, 1.5, float("nan")])
def test_probability_out_of_range_is_refused(lib, p):
    a = P16
    _refused(lib.bg_dropout_fwd(L.BG_F32, 8, p, 0, 0, a, None, a, None), "p must")
    _refused(lib.bg_dropout_bwd(8, p, 0, 0, a, a, 0, None), "p must")
    _refused(lib.bg_embed_fwd(L.BG_F32, 8, 64, 9, a, a, 1.0, p, 0, 0, a, None), "p must")
    _refused(lib.bg_embed_bwd(8, 64, 9, a, a, 1.0, p, 0, 0, a, 0, a, 1 << 30, None), "p must")


@pytest.mark.parametrize("n,H,V,word", [(-1, 64, 9, "n must"), ((1 << 30) + 1, 64, 9, "n must"),
                                        (8, 48, 9, "H must"), (8, 0, 9, "H must"),
                                        (8, 288, 9, "H must"), (8, 64, 0, "V must"),
                                        (8, 64, (1 << 24) + 1, "V must")])
def test_shapes_out_of_range_are_refused(lib, n, H, V, word):
    a = P16
    _refused(lib.bg_embed_fwd(L.BG_F32, n, H, V, a, a, 1.0, 0.0, 0, 0, a, None), word)
    _refused(lib.bg_embed_bwd(n, H, V, a, a, 1.0, 0.0, 0, 0, a, 0, a, 1 << 40, None), word)
    _refused(lib.bg_xent_fwd(L.BG_F32, n, H, V, a, a, a, a, a, a, 1 << 40, None), word)
    _refused(lib.bg_xent_bwd(L.BG_F32, n, H, V, a, a, a, a, a, L.BG_F32, a, a, 0, a, 1 << 40, None),
             word)
    assert lib.bg_embed_workspace_bytes(n, H, V) == 0
    assert lib.bg_xent_workspace_bytes(L.BG_BF16, n, H, V, L.BG_OP_XENT_FWD) == 0


def test_pointers_types_and_flags_are_checked(lib):
    a, odd = P16, P16 + 8
    _refused(lib.bg_dropout_fwd(7, 8, 0.1, 0, 0, a, None, a, None), "dtype")
    _refused(lib.bg_dropout_fwd(L.BG_F32, -1, 0.1, 0, 0, a, None, a, None), "n < 0")
    _refused(lib.bg_dropout_fwd(L.BG_F32, 8, 0.1, 0, 0, None, None, a, None), "x is NULL")
    _refused(lib.bg_dropout_fwd(L.BG_F32, 8, 0.1, 0, 0, a, odd, a, None), "residual not 16-byte")
    _refused(lib.bg_dropout_bwd(8, 0.1, 0, 0, a, a, L.BG_ACCUM, None), "BG_ACCUM")
    _refused(lib.bg_dropout_bwd(8, 0.1, 0, 0, a, a, 4, None), "flags")
    _refused(lib.bg_embed_fwd(5, 8, 64, 9, a, a, 1.0, 0.0, 0, 0, a, None), "dtype")
    _refused(lib.bg_embed_fwd(L.BG_F32, 8, 64, 9, a, odd, 1.0, 0.0, 0, 0, a, None), "table not")
    _refused(lib.bg_embed_bwd(8, 64, 9, a, a, 1.0, 0.0, 0, 0, a, 2, a, 1 << 30, None), "flags")
    _refused(lib.bg_embed_bwd(8, 64, 9, a, a, 1.0, 0.0, 0, 0, a, 0, a, 16, None), "workspace",
             code=-2)
    need = lib.bg_xent_workspace_bytes(L.BG_F32, 8, 64, 9, L.BG_OP_XENT_FWD)
    _refused(lib.bg_xent_fwd(L.BG_F32, 8, 64, 9, a, a, a, a, a, a, need - 1, None), "workspace",
             code=-2)
    _refused(lib.bg_xent_fwd(L.BG_F32, 8, 64, 9, a, None, a, a, a, a, 1 << 30, None), "W is NULL")
    big = 1 << 40
    bwd = lib.bg_xent_bwd
    _refused(bwd(L.BG_F32, 8, 64, 9, a, a, a, a, a, L.BG_BF16, a, a, 0, a, big, None), "fp32")
    _refused(bwd(L.BG_BF16, 8, 64, 9, a, a, a, a, a, L.BG_BF16, a, a, 1, a, big, None), "BG_ACCUM")
    _refused(bwd(L.BG_BF16, 8, 64, 9, a, a, a, a, a, L.BG_F32, None, None, 0, a, big, None), "dX and")
    _refused(bwd(L.BG_BF16, 8, 64, 9, a, a, a, a, a, 3, a, a, 0, a, big, None), "dtype")
    assert lib.bg_xent_workspace_bytes(L.BG_F32, 8, 64, 9, L.BG_OP_READOUT) == 0


def test_nothing_to_do_is_done_without_a_device(lib):
    assert lib.bg_dropout_fwd(L.BG_BF16, 0, 0.5, 1, 2, None, None, None, None) == 0
    assert lib.bg_dropout_bwd(0, 0.5, 1, 2, None, None, 0, None) == 0
    assert lib.bg_embed_fwd(L.BG_BF16, 0, 64, 9, None, None, 1.0, 0.0, 0, 0, None, None) == 0
    assert lib.bg_xent_fwd(L.BG_BF16, 0, 64, 9, None, P16, None, None, None, None, 0, None) == 0


def test_binding_checks_types_and_shapes():
    import torch
    x = torch.zeros(8)
    with pytest.raises(ValueError, match="x must have"):
        L.dropout_fwd("bf16", x, x, 0.1, 0, 0)
    with pytest.raises(ValueError, match="CUDA tensor"):
        L.dropout_fwd("f32", x, x, 0.1, 0, 0)
    with pytest.raises(ValueError, match="ids must be"):
        L.embed_fwd("f32", torch.zeros(3), torch.zeros(5, 64), torch.zeros(3, 64))
    with pytest.raises(ValueError, match="CUDA tensor"):
        L.embed_bwd(torch.zeros(0, dtype=torch.int32), torch.zeros(4, 64), torch.zeros(5, 64), x)


def test_workspaces_grow_with_the_work(lib):
    assert 0 < lib.bg_embed_workspace_bytes(0, 64, 9)
    assert lib.bg_embed_workspace_bytes(1000, 64, 9) < lib.bg_embed_workspace_bytes(100000, 64, 9)
    # nothing in them grows with n x V
    n, H, V = 1 << 20, 256, 1 << 20
    for dt in (L.BG_F32, L.BG_BF16):
        for op in (L.BG_OP_XENT_FWD, L.BG_OP_XENT_BWD):
            assert 0 < lib.bg_xent_workspace_bytes(dt, n, H, V, op) < 64 * H * (n + V)


def test_every_barrier_of_the_cross_entropy_kernels_is_initialised():
    """Each kernel of xent.cu initialises exactly the mbarriers that its struct declares and that it
    waits on or signals."""
    import os
    import re
    src = open(os.path.join(os.path.dirname(L.LIB_PATH), "csrc", "xent.cu")).read()
    kernels = re.findall(r"\n    k_xent_(fwd|bwd)\(const __grid_constant__.*?\n}\n", src, flags=re.S)
    assert kernels == ["fwd", "bwd"]
    for m in re.finditer(r"struct (Fwd|Bwd)Bars \{\s*uint64_t ([^;]*);", src):
        fields = {f.split("[")[0].strip() for f in m.group(2).split(",")}
        body = re.search(r"\n    k_xent_" + m.group(1).lower() + r"\(const __grid.*?\n}\n", src,
                         flags=re.S).group(0)
        init = set(re.findall(r"mbar_init\(&bars->(\w+)", body))
        used = set(re.findall(r"&bars->(\w+)", body)) - {"tmem", "abort"}
        assert init == fields == used, (fields, init, used)


def test_register_shares_add_up_to_the_launch():
    """setmaxnreg moves registers that the launch owns: four warpgroups of the epilogue and one of the others
    share the 640 x 96 of the backward's block (65536 / 640, rounded down to a multiple of 8)."""
    import os
    import re
    src = open(os.path.join(os.path.dirname(L.LIB_PATH), "csrc", "xent.cu")).read()
    dec = set(re.findall(r"setmaxnreg\.dec\.sync\.aligned\.u32 (\d+)", src))
    inc = set(re.findall(r"setmaxnreg\.inc\.sync\.aligned\.u32 (\d+)", src))
    assert len(dec) == len(inc) == 1
    assert "kBwdThreads = 640" in src
    assert 128 * int(dec.pop()) + 512 * int(inc.pop()) <= 640 * 96


def test_the_workspace_holds_what_a_call_takes_on_any_device(lib):
    """The cross entropy's kernels keep partial results for each of their CTAs, as many as the device has
    SMs: never more of them than the reported size has room for, and CTAs for both gradients even on a
    single SM."""
    import ctypes
    ctas, used = lib["_ZN2bg9xent_ctasEi"], lib["_ZN2bg12xent_ws_usedEiliiiii"]
    used.restype = ctypes.c_size_t
    used.argtypes = [ctypes.c_int, ctypes.c_int64] + [ctypes.c_int] * 5
    assert ctas(152) == 152
    for sms in (1, 2, 3, 18, 148, 152, 153, 160, 304, 1000):
        assert 2 <= ctas(sms) <= max(2, sms)
        for dt in (L.BG_F32, L.BG_BF16):
            for n, H, V in ((1, 32, 1), (700, 256, 5000), (100001, 96, 777)):
                for op, backward in ((L.BG_OP_XENT_FWD, 0), (L.BG_OP_XENT_BWD, 1)):
                    for grad_bf16 in (0, 1) if dt == L.BG_BF16 else (0,):
                        assert used(dt, n, H, V, backward, grad_bf16, sms) <= \
                            lib.bg_xent_workspace_bytes(dt, n, H, V, op)


def test_gradients_without_rows_are_not_refused(lib):
    """A tensor of no rows has no address: the gradient of the states alone is then nothing to do, and one
    that is added to is left as it is."""
    for grad in (L.BG_F32, L.BG_BF16):
        assert lib.bg_xent_bwd(L.BG_BF16, 0, 64, 9, None, P16, None, None, None, grad, None, None, 0, None,
                               0, None) == 0
    assert lib.bg_xent_bwd(L.BG_F32, 0, 64, 9, None, P16, None, None, None, L.BG_F32, None, P16, L.BG_ACCUM,
                           None, 0, None) == 0
    assert lib.bg_embed_bwd(0, 64, 9, None, None, 1.0, 0.0, 0, 0, P16, L.BG_ACCUM, None, 0, None) == 0


class _Elsewhere:
    """What the binding reads of a CUDA tensor, on a device of choice."""

    def __init__(self, device, dtype, *shape):
        self.device_index, self.dtype, self.shape, self.is_cuda = device, dtype, shape, True

    def numel(self):
        n = 1
        for m in self.shape:
            n *= m
        return n

    element_size = data_ptr = lambda self: P16
    is_contiguous = lambda self: True
    get_device = lambda self: self.device_index


def test_tensors_of_another_device_are_refused(monkeypatch):
    """The library launches on the current device: a tensor elsewhere is refused by name, before anything
    is launched, whichever of a call's tensors it is."""
    import torch
    monkeypatch.setattr(L, "_current_device", lambda: 0)
    f, i = torch.float32, torch.int32
    n, V, H = 6, 9, 64

    args = {"x": (f, n), "y": (f, n), "residual": (f, n), "dy": (f, n), "dx": (f, n), "ids": (i, n),
            "table": (f, V, H), "out": (f, n, H), "dout": (f, n, H), "dtable": (f, V, H),
            "ws": (f, 1 << 20), "X": (f, n, H), "W": (f, V, H), "target": (i, n), "loss": (f, n),
            "lse": (f, n), "dloss": (f, n), "dX": (f, n, H), "dW": (f, V, H)}
    calls = [
        ("x y residual", lambda x, y, residual: L.dropout_fwd("f32", x, y, 0.1, 1, 2, residual)),
        ("dy dx", lambda dy, dx: L.dropout_bwd(dy, dx, 0.1, 1, 2)),
        ("ids table out", lambda *t: L.embed_fwd("f32", *t)),
        ("ids dout dtable ws", lambda *t: L.embed_bwd(*t)),
        ("X W target loss lse ws", lambda *t: L.xent_fwd("f32", *t)),
        ("X W target lse dloss dX dW ws", lambda *t: L.xent_bwd("f32", *t[:5], "f32", *t[5:])),
    ]
    for names, call in calls:
        for away in names.split():
            with pytest.raises(ValueError, match=f"^{away} is on cuda:1, the current device is cuda:0"):
                call(*(_Elsewhere(int(name == away), *args[name]) for name in names.split()))
