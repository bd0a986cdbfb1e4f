"""Gradients of sequences of which a mask leaves a few states: D = rowsum(dO O)
must not carry the rounding of O, whose error dP - D would keep where O is one
state, or the average of a few.  As exact as for the same states packed into a
short sequence."""
import pytest
import torch

from attn_util import F, HALF, U
from paper_2608_01528_amd import gramspace as gs
from test_gpu_cross_attention import BF16, F32, agree, ints, problem, whole

pytestmark = pytest.mark.gpu


def one_state(B, Lk):
    """A mask that leaves one state of each sequence: first, last and others."""
    mask = torch.zeros(B, Lk, dtype=torch.bool, device="cuda")
    for b in range(B):
        mask[b, (0, Lk - 1, Lk // 2, min(64, Lk - 1))[b % 4]] = True
    return mask


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [(4, 40, 200, 2, 1, 64), (4, 1, 3000, 8, 2, 128), (4, 130, 777, 4, 2, 96), (4, 9, 129, 2, 2, 33),
                                  (33, 200, 300, 16, 8, 64)], ids=str)
def test_one_live_state_has_no_gradient(size, dtype):
    """P is 1 and dS = dP - D is 0, within the rounding of two fp32 sums of the
    same products in different orders."""
    Q, K, V, dO = problem(*size, dtype)
    got = whole(Q, K, V, dO, mask=one_state(size[0], size[2]))
    reach = float(dO.float().abs().sum(-1).max() * V.float().abs().max())
    assert float(got["dQ"].float().abs().max()) <= 64 * 2.0 ** -23 * reach * float(K.float().abs().max())
    rows = size[1] * (size[3] // size[4])
    assert float(got["dK"].float().abs().max()) <= rows * 64 * 2.0 ** -23 * reach * float(Q.float().abs().max())


def gradient_bounds(q, k, v, d, scale, half):
    """dQ and dK of one head over its live states in 64 bits, with bounds where D
    is formed in fp32 as sum_j P_j dP_j: D is off by what each P_j (the factor
    1 + e) and dP_j are, and by the sums' rounding."""
    q, k, v, d = (t.cpu().double() for t in (q, k, v, d))
    n, Dh = k.shape
    S = scale * (q @ k.t())
    lse = torch.logsumexp(S, 1)
    P = torch.exp(S - lse[:, None])
    slip = (Dh + 4) * U * scale * (q.abs() @ k.abs().t()) + 4 * U * S.abs()
    e = torch.expm1(2 * slip.amax(1) + 8 * U + 3 * U * lse.abs())[:, None]
    dP, adP = d @ v.t(), d.abs() @ v.abs().t()
    D = (P * dP).sum(1, keepdim=True)
    tol_dP = (Dh + 2) * U * adP
    tol_D = (P * (1 + e) * tol_dP + P * dP.abs() * e).sum(1, keepdim=True) + (2 * n + 64) * U * (P * dP.abs()).sum(1, keepdim=True)
    g = P * (dP - D)
    tol = P * (1 + e) * (tol_dP + tol_D + 2 * U * (dP.abs() + D.abs())) + g.abs() * e
    tol = tol + (half + 2 * U) * (g.abs() + tol) + 2 * F
    return (scale * (g @ k), scale * (tol @ k.abs() + 2 * n * U * (g.abs() @ k.abs()))), \
           (scale * (g.t() @ q), scale * (tol.t() @ q.abs() + 2 * len(q) * U * (g.abs().t() @ q.abs())))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("live", [2, 5, 31, 32])
@pytest.mark.parametrize("size", [(2, 70, 1000, 2, 2, 64), (3, 5, 333, 3, 3, 80), (2, 33, 90, 2, 2, 128)], ids=str)
def test_few_live_states(size, live, dtype):
    B, Lq, Lk, H, _, Dh = size
    Q, K, V, dO = problem(*size, dtype, factor=2.0)
    mask = torch.zeros(B, Lk, dtype=torch.bool, device="cuda")
    for b in range(B):
        at = torch.randperm(Lk, generator=torch.Generator().manual_seed(b + live))[:live]
        mask[b, at.cuda()] = True
    got = agree(Q, K, V, dO, mask=mask)
    half, scale = HALF[dtype], Dh ** -0.5
    for b in range(B):
        at = torch.nonzero(mask[b])[:, 0]
        for h in range(H):
            for name, rows, (value, bound) in zip(("dQ", "dK"), (slice(None), at), gradient_bounds(
                    Q[b, :, h], K[b, at, h], V[b, at, h], dO[b, :, h], scale, half)):
                off = (got[name][b, rows, h].cpu().double() - value).abs()
                bound = bound + (half + 2 * U) * (value.abs() + bound) + F
                assert (off <= bound).all(), (name, b, h, float((off / bound).max()))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_on_either_side_of_few(dtype):
    """Numbers of live states around the tile's, lengths and empty masks beside
    them, and the same bits from every replay."""
    B, Lq, Lk, Hq, Hkv, Dh = 8, 37, 500, 4, 2, 64
    Q, K, V, dO = problem(B, Lq, Lk, Hq, Hkv, Dh, dtype)
    mask = torch.zeros(B, Lk, dtype=torch.bool, device="cuda")
    for b, n in enumerate((0, 31, 32, 33, 63, 64, 65, 130)):
        mask[b, 7: 7 + 3 * n: 3] = True
    for kw in ({}, {"klen": ints(500, 100, 250, 70, 64, 333, 1, 0)}, {"qlen": ints(37, 0, 1, 36, 37, 5, 37, 2)}):
        first = agree(Q, K, V, dO, mask=mask, **kw)
        again = whole(Q, K, V, dO, mask=mask, **kw)
        for n in first:
            assert torch.equal(first[n], again[n]), n


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_captured_with_masks_that_change(dtype):
    """A captured step replayed with few live states, none, and many."""
    B, Lq, Lk = 2, 40, 400
    Q, K, V, dO = problem(B, Lq, Lk, 4, 2, 64, dtype)
    mask = torch.ones(B, Lk, dtype=torch.bool, device="cuda")
    whole(Q, K, V, dO, mask=mask)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = whole(Q, K, V, dO, mask=mask)
    for every in (200, 1, 13, 1000, 7, 3):
        mask.copy_((torch.arange(Lk, device="cuda")[None] % every == 2 % every).repeat(B, 1))
        if every == 1000:
            mask[1] = False
        g.replay()
        torch.cuda.synchronize()
        eager = agree(Q, K, V, dO, mask=mask)
        torch.cuda.synchronize()
        for n in eager:
            assert torch.equal(got[n], eager[n]), (every, n)
