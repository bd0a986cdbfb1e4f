"""The operators of a paged cache as a program runs them: steps of pages and
slots, stored states, attention, drafts verified and taken back, requests that
end and begin, against histories that the host keeps."""
import random

import numpy as np
import pytest
import torch

import attn_util
import paged_util
from paper_2608_01528_amd import gramspace as gs

pytestmark = pytest.mark.gpu
DEV = "cuda"
i32 = torch.int32


class Server:
    """The state of a serving program: tables, lengths and a cache, updated in place."""

    def __init__(self, B, page, pages, width, Hq, Hkv, Dh, dtype, rows):
        self.B, self.page, self.pages, self.rows = B, page, pages, rows
        self.Hq, self.Hkv, self.Dh, self.dtype = Hq, Hkv, Dh, dtype
        self.table = torch.full((B, width), -1, dtype=i32, device=DEV)
        self.length = torch.zeros(B, dtype=i32, device=DEV)
        self.free = torch.randperm(pages, device=DEV).to(i32)
        self.nfree = torch.tensor([pages], dtype=i32, device=DEV)
        self.add = torch.zeros(B, dtype=i32, device=DEV)
        self.qoff = torch.zeros(B + 1, dtype=i32, device=DEV)
        self.slots = torch.zeros(rows, dtype=torch.int64, device=DEV)
        self.added = torch.zeros(B, dtype=i32, device=DEV)
        nan = float("nan")      # what was never stored
        self.Kc, self.Vc = (torch.full((pages, page, Hkv, Dh), nan, dtype=dtype, device=DEV) for _ in range(2))
        self.K, self.V = (torch.zeros(rows, Hkv, Dh, device=DEV) for _ in range(2))
        self.Q = torch.zeros(rows, Hq, Dh, dtype=dtype, device=DEV)
        self.O, self.lse = torch.zeros_like(self.Q), torch.zeros(rows, Hq, device=DEV)

    def plan(self):
        gs.gs_paged_plan(self.length, self.add, self.table, self.free, self.nfree, page=self.page, rows=self.rows,
                         length_out=self.length, nfree_out=self.nfree, qoff_out=self.qoff, slots_out=self.slots,
                         added_out=self.added)

    def step(self, **kw):
        self.plan()
        gs.gs_paged_store(self.K, self.V, self.slots, self.Kc, self.Vc)
        gs.gs_paged_attention(self.Q, self.Kc, self.Vc, self.table, self.length, qoff=self.qoff, out=self.O, lse_out=self.lse,
                              **kw)

    def draw(self):
        for x in (self.K, self.V, self.Q):
            x.normal_()


def check(s, hist, n, window, sinks):
    """Rows of the step against their requests' histories."""
    off = s.qoff.tolist()
    for b in range(s.B):
        k = len(hist[b][0])
        for i in range(n[b]):
            j = paged_util.seen(k - n[b] + i, k, window, sinks)
            K, V = (torch.stack([h[x] for x in j])[None] for h in hist[b])
            r = off[b] + i
            ref = attn_util.reference(s.Q[None, r: r + 1], K, V)
            attn_util.check(s.O[None, r: r + 1], ref, "O")
            attn_util.check(s.lse[r][None, :, None], ref, "lse")


def consistent(s, hist):
    """Every page is free or one request's, once; tables name the pages of the lengths."""
    lens = [len(h[0]) for h in hist]
    assert s.length.tolist() == lens
    held = [-(-x // s.page) for x in lens]
    mine = [p for row, h in zip(s.table.tolist(), held) for p in row[:h]]
    spare = s.free.tolist()[: int(s.nfree)]
    assert sorted(mine + spare) == list(range(s.pages))


def keep(s, hist, n):
    """The rows' states into the histories, as the cache rounds them."""
    off, K, V = s.qoff.tolist(), s.K.to(s.dtype).cpu(), s.V.to(s.dtype).cpu()
    for b, a in enumerate(s.added.tolist()):
        assert a in (0, n[b]) or n[b] < 0
        for i in range(a):
            hist[b][0].append(K[off[b] + i])
            hist[b][1].append(V[off[b] + i])


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pages", [45, 18])
def test_steps(pages, dtype, window, sinks, captured):
    rng = random.Random(5)
    B, most, M = 6, 40, 50
    s = Server(B, page=8, pages=pages, width=12, Hq=4, Hkv=2, Dh=32, dtype=dtype, rows=B * most)
    hist = [([], []) for _ in range(B)]
    kw = {"max_new": most, "max_len": 96, "window": window, "sinks": sinks}
    graph = None
    if captured:        # warmed up, captured and replayed with nothing to do first: the state stays as it is
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s.step(**kw)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.step(**kw)
    refused = 0
    for turn in range(12):
        n = []
        for b in range(B):
            k = len(hist[b][0])
            if k and rng.random() < 0.15:
                n.append(-10**9)                    # ends
            elif k == 0:
                n.append(rng.choice([0, 1, 9, most]) if turn else most)
            else:
                n.append(rng.choice([1, 1, 4, 5]))  # a token, or drafts
        s.add.copy_(torch.tensor(n, dtype=i32))
        s.draw()
        if graph:
            graph.replay()
        else:
            s.step(**kw)
        torch.cuda.synchronize()
        for b in range(B):
            if n[b] < 0:
                hist[b][0].clear(), hist[b][1].clear()
        keep(s, hist, n)
        consistent(s, hist)
        got = s.added.tolist()
        refused += sum(a > 0 and g == 0 for a, g in zip(n, got))
        check(s, hist, got, window, sinks)
        # drafts of the requests that got their rows: some taken, the rest given back
        off = s.qoff.tolist()
        N = off[-1]
        if not N:
            continue
        P = torch.softmax(torch.randn(N, M, device=DEV) * 2, 1)
        D = torch.softmax(P.log() + 0.5 * torch.randn(N, M, device=DEV), 1)
        drafted = torch.multinomial(D, 1)[:, 0].to(i32)
        u, v = torch.rand(N, device=DEV), torch.rand(B, device=DEV)
        acc, entry, entries = gs.gs_verify(P, drafted, u, v, s.qoff, Q=D, entries=True)
        want = paged_util.verify(P.cpu().numpy(), D.cpu().numpy(), drafted.tolist(), u.cpu().numpy(), v.cpu().numpy(), off)
        assert acc.tolist() == want[0] and entry.tolist() == want[1] and entries.tolist() == want[2]
        back = [-(got[b] - 1 - want[0][b]) if got[b] and got[b] < most else 0 for b in range(B)]
        s.add.copy_(torch.tensor(back, dtype=i32))
        s.plan()
        for b in range(B):
            if back[b]:
                del hist[b][0][back[b]:], hist[b][1][back[b]:]
        torch.cuda.synchronize()
        consistent(s, hist)
    assert refused > 0 or pages == 45       # (the first step's prompts ask for 30)
    assert not np.isnan(s.O.float().cpu().numpy()).any()
