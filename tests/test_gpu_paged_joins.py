"""Histories that are cut into parts, put together by a thread for few values or by
a work-group for a row or a piece of it: each side of the rules between them."""
import pytest
import torch

import attn_util
import paged_util
from paper_2608_01528_amd import gramspace as gs

pytestmark = pytest.mark.gpu
DEV = "cuda"


# requests, rows a request, query heads over heads of keys, values, states: from 8 parts a
# request to some 500, 1 to 32 rows of a head
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,new,Hq,Hkv,Dh,Lk", [(4, 1, 16, 4, 128, 9000), (4, 4, 16, 4, 128, 9000), (2, 8, 8, 2, 64, 12000),
                                                (1, 8, 4, 1, 80, 20000), (1, 1, 4, 2, 128, 30000), (16, 4, 16, 8, 64, 2500),
                                                (3, 5, 6, 2, 96, 7001)])
def test_joins(B, new, Hq, Hkv, Dh, Lk, dtype):
    page = 32
    g = torch.Generator(device=DEV)
    g.manual_seed(B + Lk)
    i32 = dict(dtype=torch.int32, device=DEV)
    k = [Lk - 97 * b for b in range(B)]
    held = -(-Lk // page)
    Kc, Vc = (torch.randn(B * held, page, Hkv, Dh, generator=g, device=DEV).to(dtype) for _ in range(2))
    table = torch.randperm(B * held, generator=g, device=DEV).to(torch.int32).view(B, held)
    Q = torch.randn(B * new, Hq, Dh, generator=g, device=DEV).to(dtype)
    klen, qoff = torch.tensor(k, **i32), torch.arange(0, B * new + 1, new, **i32)
    O, lse = gs.gs_paged_attention(Q, Kc, Vc, table, klen, qoff, max_new=new, max_len=Lk, lse=True)
    for b in sorted({0, B - 1}):
        r = slice(b * new, b * new + new)
        ref, _ = paged_util.attention(Q[r], Kc, Vc, table[b: b + 1], klen[b: b + 1], torch.tensor([0, new], **i32))
        attn_util.check(O[r], ref, "O")
        attn_util.check(lse[r], ref, "lse")
    again = gs.gs_paged_attention(Q, Kc, Vc, table, klen, qoff, max_new=new, max_len=Lk, lse=True)
    assert torch.equal(O, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B", [2, 16, 70])
def test_one_long_history_among_short_ones(B, dtype):
    page, Hq, Hkv, Dh, new = 64, 4, 1, 64, 3
    g = torch.Generator(device=DEV)
    g.manual_seed(B)
    i32 = dict(dtype=torch.int32, device=DEV)
    k = [0 if b % 5 == 1 else 10 + b for b in range(B)]
    k[B // 2] = 40000
    n = [0 if b % 7 == 3 else new - b % 2 for b in range(B)]
    n[B // 2] = new
    held = [-(-x // page) for x in k]
    pages = sum(held)
    Kc, Vc = (torch.randn(pages, page, Hkv, Dh, generator=g, device=DEV).to(dtype) for _ in range(2))
    order, table = torch.randperm(pages, generator=g, device=DEV).to(torch.int32), torch.full((B, max(held)), -1, **i32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = order[at: at + h]
        at += h
    qoff = torch.tensor([sum(n[:b]) for b in range(B + 1)], **i32)
    Q = torch.randn(sum(n), Hq, Dh, generator=g, device=DEV).to(dtype)
    klen = torch.tensor(k, **i32)
    O, lse = gs.gs_paged_attention(Q, Kc, Vc, table, klen, qoff, max_new=new, lse=True)
    ref, _ = paged_util.attention(Q, Kc, Vc, table, klen, qoff)
    attn_util.check(O, ref, "O")
    attn_util.check(lse, ref, "lse")
