"""Refusals of gs_cross_attention, gs_cross_attention_grad and gs_sample: every
check runs on the host, so fake addresses reach no kernel (a call that passes
them ends with the missing device, or does nothing)."""
import ctypes
import struct

import pytest
import torch

from paper_2608_01528_amd import gramspace as gs

NAMES = ["B", "Lq", "Lk", "Hq", "Hkv", "Dh", "qlen", "klen", "mask", "ldm", "scale"]
SEQS = ["Q", "K", "V", "O"]
GRADS = ["dO", "dQ", "dK", "dV"]


@pytest.fixture(scope="module")
def L():
    return gs.lib()


class Problem:
    """A valid problem: B 2, Lq 3, Lk 5, 4 heads over 2, 64 values, bf16, far
    apart in memory."""

    def __init__(self, **change):
        self.v = {"B": 2, "Lq": 3, "Lk": 5, "Hq": 4, "Hkv": 2, "Dh": 64, "qlen": 0, "klen": 0, "mask": 0, "ldm": 5,
                  "scale": 0.125, "lse": 0x70000000}
        for i, n in enumerate(SEQS + GRADS):
            q = n in ("Q", "O", "dO", "dQ")
            self.v[n] = (0x10000000 + 0x1000000 * i, (3 * 4 if q else 5 * 2) * 64, (4 if q else 2) * 64, 64)
        self.v.update(change)

    def pack(self):
        v = self.v
        return gs._ATTN.pack(*[v[n] for n in NAMES], *[x for n in SEQS for x in v[n]], v["lse"],
                             *[x for n in GRADS for x in v[n]])


def fwd(L, p, t=gs.GS_BF16, ws=0x90000000, n=1 << 30):
    return L.gs_cross_attention(p.pack(), t, ws, n, None)


def grad(L, p, t=gs.GS_BF16, ws=0x90000000, n=1 << 30):
    return L.gs_cross_attention_grad(p.pack(), t, ws, n, None)


def both(L, p, t=gs.GS_BF16):
    return fwd(L, p, t), grad(L, p, t)


def say(L):
    return L.gs_last_error().decode()


@pytest.mark.skipif(torch.cuda.is_available(), reason="fake addresses")
def test_valid_problems_end_with_the_missing_device(L):
    dev = (gs.GS_ERR_DEVICE,) * 2
    assert both(L, Problem()) == dev
    assert both(L, Problem(), gs.GS_F32) == dev
    assert both(L, Problem(K=(0x11000000, 0, 128, 64))) == dev          # states shared by all sequences
    assert both(L, Problem(Lk=0)) == dev
    assert both(L, Problem(scale=-3.0)) == dev
    assert both(L, Problem(Dh=1)) == dev and both(L, Problem(Dh=63)) == dev
    assert both(L, Problem(Q=(0x10000000, 64, 128, 999999))) == dev     # an input's rows may overlap
    assert L.gs_sample(0x1000, gs.GS_F32, 2, 5, 5, 0x2000, None, 0x3000, None, None, None, 0, None) == gs.GS_ERR_DEVICE
    assert L.gs_sample(0x1000, gs.GS_BF16, 2, 70000, 70000, 0x800000, None, 0x900000, 0xa00000, 0xb00000,
                       0x10000000, 1 << 30, None) == gs.GS_ERR_DEVICE


def test_nothing_to_do(L):
    z = (0, 0, 0, 0)
    nothing = {n: z for n in SEQS + GRADS}
    assert both(L, Problem(B=0, lse=0, **nothing)) == (gs.GS_OK,) * 2
    assert both(L, Problem(Lq=0, Lk=0, lse=0, **nothing)) == (gs.GS_OK,) * 2
    assert L.gs_sample(None, gs.GS_F32, 0, 5, 5, None, None, None, None, None, None, 0, None) == gs.GS_OK


@pytest.mark.parametrize("change", [
    {"B": -1}, {"Lq": -1}, {"Lk": -2}, {"Hq": 0}, {"Hkv": 0}, {"Hq": 3}, {"Dh": 0}, {"Dh": 129}, {"B": 1 << 31},
    {"Lq": 1 << 62}, {"Lk": 1 << 40}, {"B": 1 << 20, "Lq": 1 << 20}, {"Hq": 1 << 30, "Hkv": 1 << 30, "B": 1 << 30},
    {"B": 1 << 22, "Lq": 1, "Lk": 1},
    {"Q": (0x10000000, -64, 256, 64)}, {"K": (0x11000000, 1 << 50, 128, 64)},
    {"mask": 0x80000000, "ldm": 4},
], ids=str)
def test_shapes_refused(L, change):
    p = Problem(**change)
    assert both(L, p) == (gs.GS_ERR_SHAPE,) * 2, say(L)
    if not {"Q", "K", "mask"} & set(change):
        assert L.gs_cross_attention_workspace(p.pack(), gs.GS_BF16) == 0
        assert L.gs_cross_attention_grad_workspace(p.pack(), gs.GS_BF16) == 0


@pytest.mark.parametrize("change", [
    {"B": 256, "K": (0x11000000, 1 << 39, 128, 64)},            # the last sequence beyond any memory
    {"mask": 0x80000000, "ldm": 1 << 60}, {"mask": 0x80000000, "ldm": (1 << 63) - 1},
    {"B": (1 << 23) - 1, "Hq": 1, "Hkv": 1, "Lq": 200},         # 2^24 work-groups
    {"B": (1 << 23) - 1, "Hq": 1, "Hkv": 1, "Lk": 200},
], ids=str)
def test_reach_and_work_groups_refused(L, change):
    assert both(L, Problem(**change)) == (gs.GS_ERR_SHAPE,) * 2, say(L)


def test_reach_of_scores_refused(L):
    for B, lds in ((1 << 30, 1 << 39), (3, 1 << 62)):
        assert L.gs_sample(0x1000, gs.GS_F32, B, 5, lds, 0x2000, None, 0x3000, None, None, None, 0, None) == gs.GS_ERR_SHAPE


@pytest.mark.parametrize("scale", [0.0, float("nan"), float("inf"), -float("inf"), 1e-31, 1e31])
def test_scales_refused(L, scale):
    assert both(L, Problem(scale=scale)) == (gs.GS_ERR_ARG,) * 2 and "scale" in say(L)


def test_types_addresses_and_workspaces_refused(L):
    assert both(L, Problem(), gs.GS_F64) == (gs.GS_ERR_DTYPE,) * 2
    assert L.gs_cross_attention(None, gs.GS_F32, None, 0, None) == gs.GS_ERR_ARG
    assert L.gs_cross_attention_grad(None, gs.GS_F32, None, 0, None) == gs.GS_ERR_ARG
    assert L.gs_cross_attention_workspace(None, gs.GS_F32) == 0
    for n in SEQS:
        v = Problem().v[n]
        assert both(L, Problem(**{n: (0,) + v[1:]})) == (gs.GS_ERR_ARG,) * 2 and n in say(L)
        assert both(L, Problem(**{n: (v[0] + 1,) + v[1:]})) == (gs.GS_ERR_ALIGN,) * 2
    for n in GRADS:
        v = Problem().v[n]
        assert grad(L, Problem(**{n: (0,) + v[1:]})) == gs.GS_ERR_ARG and n in say(L)
    for n in ("qlen", "klen", "lse"):
        assert both(L, Problem(**{n: 0x80000002})) == (gs.GS_ERR_ALIGN,) * 2
    assert grad(L, Problem(lse=0)) == gs.GS_ERR_ARG
    p = Problem().pack()
    need = L.gs_cross_attention_grad_workspace(p, gs.GS_BF16)
    assert need >= 2 * 3 * 4 * 4
    assert L.gs_cross_attention_grad(p, gs.GS_BF16, None, need, None) == gs.GS_ERR_WORKSPACE
    assert L.gs_cross_attention_grad(p, gs.GS_BF16, 0x90000000, need - 1, None) == gs.GS_ERR_WORKSPACE
    assert L.gs_cross_attention_grad(p, gs.GS_BF16, 0x90000008, need, None) == gs.GS_ERR_ALIGN
    long = Problem(Lq=1, Lk=1 << 16, K=(1 << 40, 1 << 24, 128, 64), V=(1 << 42, 1 << 24, 128, 64)).pack()
    need = L.gs_cross_attention_workspace(long, gs.GS_BF16)
    assert need > 0
    assert L.gs_cross_attention(long, gs.GS_BF16, None, need, None) == gs.GS_ERR_WORKSPACE
    assert L.gs_cross_attention(long, gs.GS_BF16, 0x90000000, need - 1, None) == gs.GS_ERR_WORKSPACE


def test_overlaps_refused(L):
    v = Problem().v
    for n in ("Q", "K", "V"):
        assert fwd(L, Problem(O=v[n][:1] + v["O"][1:])) == gs.GS_ERR_ARG and "overlaps" in say(L)
    assert fwd(L, Problem(lse=v["Q"][0])) == gs.GS_ERR_ARG
    assert fwd(L, Problem(qlen=v["O"][0])) == gs.GS_ERR_ARG
    assert fwd(L, Problem(mask=v["O"][0])) == gs.GS_ERR_ARG
    for n in SEQS + ["dO"]:
        assert grad(L, Problem(dK=v[n][:1] + v["dK"][1:])) == gs.GS_ERR_ARG and "overlaps" in say(L)
    assert grad(L, Problem(dV=v["dK"])) == gs.GS_ERR_ARG
    assert grad(L, Problem(), ws=v["dQ"][0]) == gs.GS_ERR_ARG
    # an output whose rows share places
    assert fwd(L, Problem(O=(v["O"][0], 0, 256, 64))) == gs.GS_ERR_SHAPE
    assert grad(L, Problem(dK=(v["dK"][0], 640, 128, 32))) == gs.GS_ERR_SHAPE
    assert grad(L, Problem(dQ=(v["dQ"][0], 256, 256, 64))) == gs.GS_ERR_SHAPE


def test_sample_refused(L):
    ok = [0x100000, gs.GS_F32, 2, 5, 5, 0x200000, None, 0x300000, 0x400000, 0x500000, None, 0, None]

    def f(*change):
        a = list(ok)
        for i, v in change:
            a[i] = v
        return L.gs_sample(*a)

    assert f((1, gs.GS_F64)) == gs.GS_ERR_DTYPE
    assert f((2, -1)) == f((3, 0)) == f((3, 1 << 31)) == f((2, 1 << 31)) == f((4, 4)) == gs.GS_ERR_SHAPE
    assert f((0, None)) == f((5, None)) == f((7, None)) == gs.GS_ERR_ARG
    assert f((0, 0x100002)) == f((5, 0x200002)) == f((7, 0x300001)) == f((8, 0x400002)) == f((9, 0x500002)) == gs.GS_ERR_ALIGN
    assert f((7, 0x100000)) == f((8, 0x300004)) == f((9, 0x200000)) == gs.GS_ERR_ARG
    for i in range(4):
        at = [0, 0, 0, 0]
        at[i] = 0x600002
        assert f((6, gs._SAMPLING.pack(*at, 1.0, 0, 1.0, 0.0))) == gs.GS_ERR_ALIGN
        at[i] = 0x300004
        assert f((6, gs._SAMPLING.pack(*at, 1.0, 0, 1.0, 0.0))) == gs.GS_ERR_ARG
    assert L.gs_sample_workspace(gs.GS_F64, 1, 100000) == 0 and L.gs_sample_workspace(gs.GS_F32, -1, 5) == 0


def test_packed_structs_match_the_header():
    class Seq(ctypes.Structure):
        _fields_ = [("p", ctypes.c_void_p), ("sb", ctypes.c_int64), ("sl", ctypes.c_int64), ("sh", ctypes.c_int64)]

    class Attn(ctypes.Structure):
        _fields_ = ([(n, ctypes.c_int64) for n in NAMES[:6]] + [(n, ctypes.c_void_p) for n in ("qlen", "klen", "mask")]
                    + [("ldm", ctypes.c_int64), ("scale", ctypes.c_double)] + [(n, Seq) for n in SEQS]
                    + [("lse", ctypes.c_void_p)] + [(n, Seq) for n in GRADS])

    class Sampling(ctypes.Structure):
        _fields_ = [(n, ctypes.c_void_p) for n in "tkpm"] + [("t1", ctypes.c_float), ("k1", ctypes.c_int32),
                                                             ("p1", ctypes.c_float), ("m1", ctypes.c_float)]

    assert ctypes.sizeof(Attn) == gs._ATTN.size and ctypes.sizeof(Sampling) == gs._SAMPLING.size
    a = Attn.from_buffer_copy(Problem(mask=0x80000000, klen=0x90000004).pack())
    assert (a.B, a.Dh, a.klen, a.mask, a.scale, a.K.p, a.K.sl, a.lse, a.dV.sb) == (
        2, 64, 0x90000004, 0x80000000, 0.125, 0x11000000, 128, 0x70000000, 640)
    s = Sampling.from_buffer_copy(gs._SAMPLING.pack(1, 2, 3, 4, 0.5, 7, 0.25, 0.125))
    assert (s.t, s.m, s.t1, s.k1, s.p1, s.m1) == (1, 4, 0.5, 7, 0.25, 0.125)
    assert struct.calcsize("P") == 8


def test_wrappers_refuse():
    f = lambda *n, dtype=torch.float32: torch.zeros(*n, dtype=dtype)  # noqa: E731
    q, k = f(2, 3, 4, 8), f(2, 5, 2, 8)
    for call in (lambda: gs.gs_cross_attention(q, k, k),                    # not on the GPU
                 lambda: gs.gs_cross_attention(q[0], k, k),
                 lambda: gs.gs_cross_attention(q, k, f(2, 5, 2, 7)),
                 lambda: gs.gs_cross_attention(q, f(3, 5, 2, 8), k),
                 lambda: gs.gs_cross_attention(q, k, k, mask=f(2, 5)),
                 lambda: gs.gs_cross_attention(q.half(), k.half(), k.half()),
                 lambda: gs.gs_sample(f(2, 3), f(2)),
                 lambda: gs.gs_sample(f(6), f(2)),
                 lambda: gs.gs_sample(f(2, 3), None)):
        with pytest.raises(ValueError):
            call()
