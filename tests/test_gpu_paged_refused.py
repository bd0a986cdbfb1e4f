"""Requests that a step's plan refuses their positions: their rows of the step stand
for none, and what the other requests get is as without them."""
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


def ints(x):
    return torch.tensor(x, dtype=i32, device=DEV)


def serving(seed, dtype, n, k, page, spare, Hq, Hkv, Dh):
    """A cache that holds k[b] states of each request, and a step that asks for n[b]
    more with `spare` free pages: the plan's results and tensors of its rows."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    held = [-(-x // page) for x in k]
    pages = sum(held) + spare
    width = max(-(-(a + b) // page) for a, b in zip(n, k))
    order = torch.randperm(pages, generator=g, device=DEV).to(i32)
    table = torch.full((len(k), width), -1, dtype=i32, device=DEV)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = order[at: at + h]
        at += h
    free, nfree = order[at:].clone() if spare else ints([-1]), ints([spare])
    rows = sum(n)
    length, _, qoff, slots, added = gs.gs_paged_plan(ints(k), ints(n), table, free, nfree, page=page, rows=rows)
    normal = lambda *s: torch.randn(*s, generator=g, device=DEV).to(dtype)  # noqa: E731
    Kc, Vc, K, V, Q = (normal(pages, page, Hkv, Dh), normal(pages, page, Hkv, Dh), normal(rows, Hkv, Dh),
                       normal(rows, Hkv, Dh), normal(rows, Hq, Dh))
    gs.gs_paged_store(K, V, slots, Kc, Vc)
    return table, length, qoff, added, Q, Kc, Vc


# tokens, drafts of up to 16 and of up to 32 packed rows, pieces of prompts; histories
# short enough for a launch of their own, and cut
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 2)])
@pytest.mark.parametrize("n,k,G", [([1, 1, 1, 1], [16, 40, 0, 33], 2), ([4, 3, 8, 1], [16, 47, 0, 32], 2), ([8, 5, 1, 8], [16, 48, 3, 31], 4),
                                   ([1, 1, 1], [4000, 3200, 5], 4), ([60, 1, 200, 3], [32, 48, 1, 300], 4)])
def test_attention(n, k, G, window, sinks, dtype):
    Hkv, Dh, page = 2, 64, 16
    seen = set()
    for spare in (0, 1, 2, 5, 40):
        table, length, qoff, added, Q, Kc, Vc = serving(spare, dtype, n, k, page, spare, G * Hkv, Hkv, Dh)
        got = added.tolist()
        seen |= {a > 0 for a in got}
        kw = dict(qoff=qoff, max_new=max(n), window=window, sinks=sinks)
        out, lse = torch.full_like(Q, 7.0), torch.full(Q.shape[:2], 7.0, device=DEV)
        gs.gs_paged_attention(Q, Kc, Vc, table, length, out=out, lse_out=lse, added=added, **kw)
        # a request that got nothing has no states for its rows
        ref, _ = paged_util.attention(Q, Kc, Vc, table, torch.where(added > 0, length, 0), qoff, window=window, sinks=sinks)
        attn_util.check(out, ref, "O")
        attn_util.check(lse, ref, "lse")
        off = qoff.tolist()
        for b, a in enumerate(got):
            r = slice(off[b], off[b + 1])
            if not a:
                assert (out[r] == 0).all() and (lse[r] == -float("inf")).all()
        if all(got):
            plain = gs.gs_paged_attention(Q, Kc, Vc, table, length, lse=True, **kw)
            assert torch.equal(plain[0], out) and torch.equal(plain[1], lse)
    assert seen == {False, True}


def test_tokens_without_offsets():
    """A row a request: those that got nothing (0, or positions taken back) see nothing."""
    B, page = 70, 16
    rng = random.Random(1)
    k = [rng.choice([0, 1, 16, 90]) for _ in range(B)]
    table, length, _, _, Q, Kc, Vc = serving(3, torch.bfloat16, [1] * B, k, page, 100, 4, 2, 64)
    added = ints([rng.choice([0, 1, 1, -3]) for _ in range(B)])
    O, lse = gs.gs_paged_attention(Q, Kc, Vc, table, length, added=added, lse=True)
    want = gs.gs_paged_attention(Q, Kc, Vc, table, length, lse=True)
    on = added > 0
    assert torch.equal(O[on], want[0][on]) and torch.equal(lse[on], want[1][on])
    assert (O[~on] == 0).all() and (lse[~on] == -float("inf")).all()


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M", [3, 200, 3000, 9000])
def test_verify(M, dtype, draft):
    g = torch.Generator(device=DEV)
    g.manual_seed(M)
    n = [1, 4, 3, 0, 80, 2, 5]
    added = [1, 0, 3, 0, 0, -2, 5]
    qoff = ints([0] + np.cumsum(n).tolist())
    N, B = sum(n), len(n)
    P, D = (torch.softmax(2 * torch.randn(N, M, generator=g, device=DEV), 1).to(dtype) for _ in range(2))
    drafted = torch.randint(0, M, (N,), generator=g, device=DEV).to(i32)
    u, v = torch.rand(N, generator=g, device=DEV) * 0.3, torch.rand(B, generator=g, device=DEV)
    Q = D if draft else None
    want = gs.gs_verify(P, drafted, u, v, qoff, Q=Q, entries=True)
    off = qoff.tolist()
    for b, a in enumerate(added):           # rows of theirs are not read
        if a <= 0:
            P[off[b]: off[b + 1]] = float("nan")
    acc, entry, entries = gs.gs_verify(P, drafted, u, v, qoff, Q=Q, entries=True, added=ints(added))
    for b, a in enumerate(added):
        r = slice(off[b], off[b + 1])
        if a > 0:
            assert acc[b] == want[0][b] and entry[b] == want[1][b] and torch.equal(entries[r], want[2][r])
        else:
            assert acc[b] == 0 and entry[b] == -1 and (entries[r] == -1).all()


def test_a_captured_step_refuses_and_serves():
    """The chain plan, store, attention, verify in one graph, replayed with other
    requests: what was refused is the plan's to say each time."""
    n, k, page, spare, M = [3, 2, 4], [16, 16, 30], 16, 2, 500
    Hkv, Dh, pages = 2, 64, 8
    table0 = ints([[0, -1, -1], [1, -1, -1], [2, 3, -1]])
    table, free, nfree = table0.clone(), ints([4, 5, 6, 7]), ints([spare])
    length, add = ints(k), ints(n)
    N, B = 9, 3
    Kc, Vc = (torch.randn(pages, page, Hkv, Dh, device=DEV) for _ in range(2))
    K, V, Q = torch.randn(N, Hkv, Dh, device=DEV), torch.randn(N, Hkv, Dh, device=DEV), torch.randn(N, 4, Dh, device=DEV)
    P = torch.softmax(torch.randn(N, M, device=DEV), 1)
    drafted, u, v = torch.zeros(N, dtype=i32, device=DEV), torch.zeros(N, device=DEV), torch.rand(B, device=DEV)

    def step():
        length1, _, qoff, slots, added = gs.gs_paged_plan(length, add, table, free, nfree, page=page, rows=N)
        gs.gs_paged_store(K, V, slots, Kc, Vc)
        O, lse = gs.gs_paged_attention(Q, Kc, Vc, table, length1, qoff=qoff, max_new=4, added=added, lse=True)
        return (added, O, lse) + gs.gs_verify(P, drafted, u, v, qoff, entries=True, added=added)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for pages_free, ask, got in ((2, [3, 2, 4], [3, 2, 0]), (0, [3, 2, 2], [0, 0, 2]), (4, [3, 2, 4], [3, 2, 4]), (1, [0, 2, 4], [0, 2, 0])):
        nfree.copy_(ints([pages_free]))
        add.copy_(ints(ask))
        K.normal_(), V.normal_(), Q.normal_()
        table.copy_(table0)
        graph.replay()
        replayed = [x.clone() for x in out]
        table.copy_(table0)
        eager = step()
        torch.cuda.synchronize()
        assert replayed[0].tolist() == got
        at = 0
        for b, (a, g) in enumerate(zip(ask, got)):
            r = slice(at, at + a)
            at += a
            for x, y in zip(replayed[1:3], eager[1:3]):
                assert torch.equal(x[r], y[r])
            assert torch.equal(replayed[5][r], eager[5][r])
            if a and not g:
                assert (replayed[1][r] == 0).all() and (replayed[2][r] == -float("inf")).all()
                assert replayed[3][b] == 0 and replayed[4][b] == -1 and (replayed[5][r] == -1).all()
            elif a:
                assert (replayed[1][r] != 0).any() and replayed[4][b] >= 0
