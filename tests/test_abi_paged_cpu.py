"""Refusals of gs_paged_plan, gs_paged_store, gs_paged_attention and gs_verify:
every check runs on the host, so fake addresses reach no kernel (a call that
passes them ends with the missing device, or does nothing)."""
import pytest
import torch

from paper_2608_01528_amd import gramspace as gs

NO_GPU = pytest.mark.skipif(torch.cuda.is_available(), reason="fake addresses")
WS = 0x700000000000


@pytest.fixture(scope="module")
def L():
    return gs.lib()


class Args:
    """A valid problem, its fields in order; fields may be changed by name."""
    order, pack, base = (), None, {}

    def __init__(self, **change):
        self.v = dict(self.base, **change)
        assert set(self.v) == set(self.base)

    def bytes(self):
        flat = []
        for n in self.order:
            x = self.v[n]
            flat += x if isinstance(x, tuple) else (x,)
        return self.pack.pack(*flat)


class Step(Args):
    order = ("B", "page", "rows", "length", "add", "length_out", "table", "width", "ldt", "free", "capacity", "nfree",
             "nfree_out", "qoff", "slots", "added")
    pack = gs._PAGED_STEP
    base = dict(B=3, page=16, rows=40, length=0x10000000, add=0x11000000, length_out=0x12000000, table=0x13000000, width=5,
                ldt=6, free=0x14000000, capacity=50, nfree=0x15000000, nfree_out=0x16000000, qoff=0x17000000,
                slots=0x18000000, added=0x19000000)

    def call(self, L, ws=WS, n=1 << 20):
        return L.gs_paged_plan(self.bytes(), ws, n, None)


class Rows(Args):
    order = ("N", "Hkv", "Dh", "pages", "page", "slots", "K", "V", "Kc", "Vc")
    pack = gs._PAGED_ROWS
    base = dict(N=7, Hkv=2, Dh=64, pages=10, page=16, slots=0x10000000, K=(0x11000000, 0, 128, 64), V=(0x12000000, 0, 128, 64),
                Kc=(0x13000000, 2048, 128, 64), Vc=(0x14000000, 2048, 128, 64))

    def call(self, L, t=gs.GS_F32, ct=gs.GS_BF16):
        return L.gs_paged_store(self.bytes(), t, ct, None)


class Attn(Args):
    order = ("B", "N", "Lq", "Lk", "Hq", "Hkv", "Dh", "pages", "page", "width", "ldt", "table", "klen", "qoff", "window",
             "sinks", "scale", "Q", "K", "V", "O", "lse")
    pack = gs._PAGED_ATTN
    base = dict(B=3, N=9, Lq=4, Lk=70, Hq=4, Hkv=2, Dh=64, pages=10, page=16, width=5, ldt=5, table=0x10000000,
                klen=0x11000000, qoff=0x12000000, window=0, sinks=0, scale=0.125, Q=(0x13000000, 0, 256, 64),
                K=(0x14000000, 2048, 128, 64), V=(0x15000000, 2048, 128, 64), O=(0x16000000, 0, 256, 64), lse=0x17000000)

    def call(self, L, t=gs.GS_BF16, ws=WS, n=1 << 30):
        return L.gs_paged_attention(self.bytes(), t, ws, n, None)


class Drafts(Args):
    order = ("B", "N", "M", "P", "ldp", "Q", "ldq", "drafted", "u", "v", "qoff", "accepted", "entry", "entries")
    pack = gs._DRAFTS
    base = dict(B=3, N=9, M=100, P=0x10000000, ldp=100, Q=0x11000000, ldq=104, drafted=0x12000000, u=0x13000000, v=0x14000000,
                qoff=0x15000000, accepted=0x16000000, entry=0x17000000, entries=0x18000000)

    def call(self, L, t=gs.GS_F32, ws=WS, n=1 << 30):
        return L.gs_verify(self.bytes(), t, ws, n, None)


EVERY = [Step, Rows, Attn, Drafts]
BIG = 2**31 - 256


@NO_GPU
@pytest.mark.parametrize("kind", EVERY)
def test_valid_problems_end_with_the_missing_device(L, kind):
    assert kind().call(L) == gs.GS_ERR_DEVICE


@pytest.mark.parametrize("kind,change", [
    (Step, dict(B=0, length=0, add=0, length_out=0, table=0, added=0)), (Step, dict(rows=0, slots=0)),
    (Step, dict(capacity=0, free=0)), (Step, dict(width=0, ldt=0, table=0)),
    (Step, dict(length_out=0x10000000)), (Step, dict(nfree_out=0x15000000)),
    (Rows, dict(Kc=(0x13000000, 4096, 128, 64), Vc=(0x13001000, 4096, 128, 64))),
    (Rows, dict(Kc=(0x13000000, 4096, 256, 128), Vc=(0x13000080, 4096, 256, 128))),
    (Attn, dict(qoff=0, N=3)), (Attn, dict(lse=0)), (Attn, dict(Lk=80)), (Attn, dict(window=2**62, sinks=2**62)),
    (Attn, dict(Lk=0, table=0)), (Attn, dict(pages=0, K=(0, 0, 0, 0), V=(0, 0, 0, 0))),
    (Drafts, dict(Q=0)), (Drafts, dict(entries=0)), (Drafts, dict(M=2**31 - 257, ldp=2**31, ldq=2**31, N=1, B=3, P=2**44, Q=2**45))])
@NO_GPU
def test_allowed(L, kind, change):
    assert kind(**change).call(L, **({"n": 1 << 40} if kind in (Step, Attn, Drafts) else {})) == gs.GS_ERR_DEVICE


@pytest.mark.parametrize("kind,change", [(Rows, dict(N=0, slots=0, K=(0, 0, 0, 0), V=(0, 0, 0, 0))),
                                         (Rows, dict(pages=0, Kc=(0, 0, 0, 0), Vc=(0, 0, 0, 0))),
                                         (Attn, dict(B=0)), (Attn, dict(N=0)), (Attn, dict(Lq=0)), (Drafts, dict(B=0, N=0))])
def test_nothing_to_do(L, kind, change):
    assert kind(**change).call(L) == gs.GS_OK


@pytest.mark.parametrize("kind,change,status", [
    (Step, dict(B=-1), gs.GS_ERR_SHAPE), (Step, dict(B=BIG), gs.GS_ERR_SHAPE), (Step, dict(page=0), gs.GS_ERR_SHAPE),
    (Step, dict(page=BIG), gs.GS_ERR_SHAPE), (Step, dict(rows=-1), gs.GS_ERR_SHAPE), (Step, dict(width=-1), gs.GS_ERR_SHAPE),
    (Step, dict(ldt=4), gs.GS_ERR_SHAPE), (Step, dict(ldt=2**46), gs.GS_ERR_SHAPE), (Step, dict(capacity=-1), gs.GS_ERR_SHAPE),
    (Step, dict(slots=0x18000004), gs.GS_ERR_ALIGN), (Step, dict(length=0x10000002), gs.GS_ERR_ALIGN),
    (Step, dict(length_out=0x10000004), gs.GS_ERR_ARG),         # not the lengths, but over them
    (Step, dict(add=0x12000000), gs.GS_ERR_ARG), (Step, dict(qoff=0x13000000), gs.GS_ERR_ARG),
    (Step, dict(nfree_out=0x14000000), gs.GS_ERR_ARG), (Step, dict(added=0x10000000), gs.GS_ERR_ARG),
    (Step, dict(slots=WS, rows=5000), gs.GS_ERR_ARG),
    (Rows, dict(N=-1), gs.GS_ERR_SHAPE), (Rows, dict(Hkv=0), gs.GS_ERR_SHAPE), (Rows, dict(Dh=0), gs.GS_ERR_SHAPE),
    (Rows, dict(page=0), gs.GS_ERR_SHAPE), (Rows, dict(pages=-1), gs.GS_ERR_SHAPE),
    (Rows, dict(N=2**30, Dh=40), gs.GS_ERR_SHAPE), (Rows, dict(slots=0), gs.GS_ERR_ARG),
    (Rows, dict(slots=0x10000004), gs.GS_ERR_ALIGN), (Rows, dict(K=(0x11000002, 0, 128, 64)), gs.GS_ERR_ALIGN),
    (Rows, dict(K=(0, 0, 128, 64)), gs.GS_ERR_ARG), (Rows, dict(Kc=(0x13000000, 2048, 128, 63)), gs.GS_ERR_SHAPE),
    (Rows, dict(Kc=(0x13000000, 0, 128, 64)), gs.GS_ERR_SHAPE), (Rows, dict(Vc=(0x14000000, -1, 128, 64)), gs.GS_ERR_SHAPE),
    (Rows, dict(Vc=(0x14000000, 2**41, 128, 64)), gs.GS_ERR_SHAPE), (Rows, dict(Kc=(0x11000000, 2048, 128, 64)), gs.GS_ERR_ARG),
    (Rows, dict(Vc=(0x13000100, 2048, 128, 64)), gs.GS_ERR_ARG), (Rows, dict(Vc=(0x13000000, 2048, 128, 64)), gs.GS_ERR_ARG),
    # side by side, but a value too near, of other strides, or over the rows that are read
    (Rows, dict(Kc=(0x13000000, 4096, 128, 64), Vc=(0x13000ffe, 4096, 128, 64)), gs.GS_ERR_ARG),
    (Rows, dict(Kc=(0x13000000, 4096, 128, 64), Vc=(0x13001000, 4096, 64, 1024)), gs.GS_ERR_ARG),
    (Rows, dict(Kc=(0x13000000, 4096, 128, 64), Vc=(0x13001000, 4096, 128, 64), K=(0x13010000, 0, 128, 64)), gs.GS_ERR_ARG),
    (Attn, dict(B=-1), gs.GS_ERR_SHAPE), (Attn, dict(N=-1), gs.GS_ERR_SHAPE), (Attn, dict(Lq=-1), gs.GS_ERR_SHAPE),
    (Attn, dict(Lk=81), gs.GS_ERR_SHAPE), (Attn, dict(Lk=-1), gs.GS_ERR_SHAPE), (Attn, dict(Hkv=3), gs.GS_ERR_SHAPE),
    (Attn, dict(Hkv=0), gs.GS_ERR_SHAPE), (Attn, dict(Hq=0), gs.GS_ERR_SHAPE), (Attn, dict(Dh=129), gs.GS_ERR_SHAPE),
    (Attn, dict(Dh=0), gs.GS_ERR_SHAPE), (Attn, dict(page=0), gs.GS_ERR_SHAPE), (Attn, dict(pages=-1), gs.GS_ERR_SHAPE),
    (Attn, dict(window=-1), gs.GS_ERR_SHAPE), (Attn, dict(sinks=-1), gs.GS_ERR_SHAPE),
    (Attn, dict(N=2**28, Lq=1), gs.GS_ERR_SHAPE), (Attn, dict(B=2**21), gs.GS_ERR_SHAPE),
    (Attn, dict(Hq=2**16, Hkv=2**16), gs.GS_ERR_SHAPE), (Attn, dict(B=2**9, Lk=2**27, page=2**25), gs.GS_ERR_SHAPE),
    (Attn, dict(qoff=0), gs.GS_ERR_SHAPE), (Attn, dict(ldt=4), gs.GS_ERR_SHAPE), (Attn, dict(ldt=2**45), gs.GS_ERR_SHAPE),
    (Attn, dict(scale=0.0), gs.GS_ERR_ARG), (Attn, dict(scale=float("nan")), gs.GS_ERR_ARG),
    (Attn, dict(scale=1e31), gs.GS_ERR_ARG), (Attn, dict(klen=0), gs.GS_ERR_ARG), (Attn, dict(table=0), gs.GS_ERR_ARG),
    (Attn, dict(table=0x10000002), gs.GS_ERR_ALIGN), (Attn, dict(lse=0x17000002), gs.GS_ERR_ALIGN),
    (Attn, dict(Q=(0, 0, 256, 64)), gs.GS_ERR_ARG), (Attn, dict(K=(0x14000001, 2048, 128, 64)), gs.GS_ERR_ALIGN),
    (Attn, dict(O=(0x16000000, 0, 255, 64)), gs.GS_ERR_SHAPE), (Attn, dict(O=(0x13000000, 0, 256, 64)), gs.GS_ERR_ARG),
    (Attn, dict(lse=0x16000000), gs.GS_ERR_ARG), (Attn, dict(O=(0x14001000, 0, 256, 64)), gs.GS_ERR_ARG),
    (Attn, dict(O=(WS, 0, 256, 64), Lk=300, width=20, ldt=20), gs.GS_ERR_ARG),
    (Drafts, dict(B=-1), gs.GS_ERR_SHAPE), (Drafts, dict(N=-1), gs.GS_ERR_SHAPE), (Drafts, dict(M=0), gs.GS_ERR_SHAPE),
    (Drafts, dict(M=BIG, ldp=BIG, ldq=BIG), gs.GS_ERR_SHAPE), (Drafts, dict(B=2**24), gs.GS_ERR_SHAPE),
    (Drafts, dict(B=2**14, M=2**22, ldp=2**22, ldq=2**22), gs.GS_ERR_SHAPE), (Drafts, dict(ldp=99), gs.GS_ERR_SHAPE),
    (Drafts, dict(ldq=99), gs.GS_ERR_SHAPE), (Drafts, dict(ldp=2**46), gs.GS_ERR_SHAPE),
    (Drafts, dict(P=0), gs.GS_ERR_ARG), (Drafts, dict(drafted=0), gs.GS_ERR_ARG), (Drafts, dict(u=0), gs.GS_ERR_ARG),
    (Drafts, dict(v=0), gs.GS_ERR_ARG), (Drafts, dict(qoff=0), gs.GS_ERR_ARG), (Drafts, dict(accepted=0), gs.GS_ERR_ARG),
    (Drafts, dict(entry=0), gs.GS_ERR_ARG), (Drafts, dict(entries=0x12000000), gs.GS_ERR_ARG),
    (Drafts, dict(entry=0x16000004), gs.GS_ERR_ARG), (Drafts, dict(u=0x13000001), gs.GS_ERR_ALIGN),
    (Drafts, dict(P=0x10000002), gs.GS_ERR_ALIGN),
] + [(Step, {n: 0}, gs.GS_ERR_ARG) for n in ("length", "add", "length_out", "table", "free", "nfree", "nfree_out", "qoff",
                                             "slots", "added")])
def test_refused(L, kind, change, status):
    assert kind(**change).call(L) == status
    assert L.gs_last_error()


def test_types(L):
    assert Rows().call(L, t=gs.GS_F64) == gs.GS_ERR_DTYPE and Rows().call(L, ct=gs.GS_F64) == gs.GS_ERR_DTYPE
    assert Attn().call(L, t=gs.GS_F64) == gs.GS_ERR_DTYPE and Attn().call(L, t=7) == gs.GS_ERR_DTYPE
    assert Drafts().call(L, t=gs.GS_F64) == gs.GS_ERR_DTYPE


def test_null_problems(L):
    for r in (L.gs_paged_plan(None, WS, 1 << 20, None), L.gs_paged_store(None, 0, 0, None),
              L.gs_paged_attention(None, 1, WS, 1 << 20, None), L.gs_verify(None, 0, WS, 1 << 20, None)):
        assert r == gs.GS_ERR_ARG
    assert L.gs_paged_attention_workspace(None, 1) == 0


def test_workspaces(L):
    """Sizes that are asked for are the sizes that are enough."""
    M = 50000
    for kind, need, change in ((Step, L.gs_paged_plan_workspace(Step(rows=5000).bytes()), dict(rows=5000)),
                               (Attn, L.gs_paged_attention_workspace(Attn(Lk=300, page=64).bytes(), gs.GS_BF16),
                                dict(Lk=300, page=64, K=(0x14000000, 8192, 128, 64), V=(0x15000000, 8192, 128, 64))),
                               (Attn, L.gs_paged_attention_workspace(Attn(Lq=9, Hq=64).bytes(), gs.GS_BF16),
                                dict(Lq=9, Hq=64, Q=(0x13000000, 0, 4096, 64), O=(0x16000000, 0, 4096, 64))),
                               (Drafts, L.gs_verify_workspace(3, M), dict(M=M, ldp=M, ldq=M, P=0x20000000, Q=0x30000000))):
        assert need > 0
        assert kind(**change).call(L, ws=None, n=0) == gs.GS_ERR_WORKSPACE
        assert kind(**change).call(L, n=need - 1) == gs.GS_ERR_WORKSPACE
        assert kind(**change).call(L, ws=WS + 8, n=need) == gs.GS_ERR_ALIGN
        if not torch.cuda.is_available():
            assert kind(**change).call(L, n=need) == gs.GS_ERR_DEVICE
    assert L.gs_verify_workspace(3, 4096) == 0 and L.gs_verify_workspace(0, M) == 0 and L.gs_verify_workspace(2**24, M) == 0
    assert L.gs_paged_plan_workspace(Step(B=-1, rows=5000).bytes()) == 0 and L.gs_paged_plan_workspace(Step().bytes()) == 0
    assert L.gs_paged_plan_workspace(None) == 0 and L.gs_paged_attention_workspace(Attn().bytes(), gs.GS_BF16) == 0
    for change in (dict(B=0), dict(N=0), dict(Lq=0), dict(Dh=129), dict(Lk=81)):
        assert L.gs_paged_attention_workspace(Attn(**change).bytes(), gs.GS_BF16) == 0
    assert L.gs_paged_attention_workspace(Attn().bytes(), gs.GS_F64) == 0


def test_binding_refuses_host_tensors():
    i = torch.zeros(3, dtype=torch.int32)
    c = torch.zeros(4, 8, 2, 16)
    for f in (lambda: gs.gs_paged_plan(i, i, i.view(3, 1), i, i[:1], page=4, rows=3),
              lambda: gs.gs_paged_store(torch.zeros(3, 2, 16), torch.zeros(3, 2, 16), torch.zeros(3, dtype=torch.int64), c, c),
              lambda: gs.gs_paged_attention(torch.zeros(3, 2, 16), c, c, i.view(3, 1), i),
              lambda: gs.gs_verify(torch.zeros(3, 5), i, torch.zeros(3), torch.zeros(2), i)):
        with pytest.raises(ValueError, match="GPU"):
            f()
