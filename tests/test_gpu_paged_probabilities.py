"""How near gs_paged_attention comes where the probabilities' rounding is all there is.

Scores are products of few terms, so nearly exact; the probabilities of two groups
of keys lie between steps of bf16, to opposite sides, and their values cancel.
The first key has the largest score, so probabilities are exp(S) on their way
into the product."""
import math

import pytest
import torch

from paper_2608_01528_amd import gramspace as gs

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16
U = 2.0**-24


def between_steps():
    """Scores in [-2, -0.5] whose exponentials are rounded down and up the most."""
    x = torch.arange(-2, -0.5, 2.0**-7, dtype=torch.float64).to(BF16).double()
    p = x.exp()
    off = (p.to(BF16).double() - p) / p
    return float(x[off.argmin()]), float(x[off.argmax()])


# rows a request: up to 16 packed ones in products of 16 x 16, up to 32 in such of 32 x 32
@pytest.mark.parametrize("new,Hq,Hkv,Dh", [(1, 1, 1, 64), (1, 8, 1, 128), (4, 4, 2, 80), (5, 4, 1, 64), (4, 16, 2, 128)])
@pytest.mark.parametrize("k", [40, 500, 3000])
def test_two_terms(new, Hq, Hkv, Dh, k):
    """Tokens and drafts in bf16: a probability is off by 2^-15 at most, of which
    O has sum p |v|; by e = 2 dS + 8 u + 3 u |lse| from scores (of those above -2:
    the others weigh 1e-21) and their sum, and sums by n u of their terms, as in
    attn_util; and the result by half its step."""
    down, up = between_steps()
    S = torch.full((k,), -50.0, dtype=torch.float64)      # (the last ones: seen by some rows only)
    n = k - new
    S[:n] = torch.where(torch.arange(n) % 2 == 0, down, up)
    S[0] = 0.0
    p = S.exp()
    w = torch.where(S == down, 1.0, torch.where(S == up, -math.exp(down - up), 0.0)).to(BF16).double()
    K, V = torch.zeros(1, k, Hkv, Dh, dtype=BF16), torch.zeros(1, k, Hkv, Dh, dtype=BF16)
    K[0, :, :, 0] = S.to(BF16)[:, None]
    V[0] = w.to(BF16)[:, None, None]
    Q = torch.zeros(new, Hq, Dh, dtype=BF16)
    Q[:, :, 0] = 1
    page = 16
    pages = -(-k // page)
    cache = [torch.zeros(pages * page, Hkv, Dh, dtype=BF16) for _ in range(2)]
    for c, x in zip(cache, (K, V)):
        c[:k] = x[0]
    Kc, Vc = (c.view(pages, page, Hkv, Dh).to(DEV) for c in cache)
    i32 = dict(dtype=torch.int32, device=DEV)
    O = gs.gs_paged_attention(Q.to(DEV), Kc, Vc, torch.arange(pages, **i32)[None], torch.tensor([k], **i32),
                              torch.tensor([0, new], **i32), max_new=new, scale=1.0).cpu().double()
    for i in range(new):
        at = slice(0, n + i + 1)
        total = p[at].sum()
        o, A = float((p[at] * w[at]).sum() / total), float((p[at] * w[at].abs()).sum() / total)
        e = 2 * ((Dh + 4) * U * 2 + 4 * U * 2) + 8 * U + 3 * U * abs(math.log(total))
        tol = A * (2.0**-15 + 2 * e + 2 * (2 * k + 64) * U)
        tol += 2.0**-8 * (abs(o) + tol)
        assert tol < 0.25 * 2.0**-8 * A         # one term may be off by more than that
        assert (O[i] - o).abs().max() <= tol, (i, float((O[i] - o).abs().max() / tol))


@pytest.mark.parametrize("new,G", [(1, 4), (5, 4), (4, 8)])
@pytest.mark.parametrize("S", [0.0, -3.0, -69.0])
def test_infinite_values_of_any_weight(new, G, S):
    """A value that is infinite makes its column infinite in the rows that see it, however little it weighs."""
    k, page, Dh = 200, 8, 64
    for value in (math.inf, -math.inf):
        Kc, Vc = torch.zeros(25, page, 1, Dh, dtype=BF16, device=DEV), torch.randn(25, page, 1, Dh, device=DEV).to(BF16)
        Kc[9, 3, 0, 0], Vc[9, 3, 0, 7] = S, value
        Q = torch.zeros(new, G, Dh, dtype=BF16, device=DEV)
        Q[:, :, 0] = 1
        i32 = dict(dtype=torch.int32, device=DEV)
        O = gs.gs_paged_attention(Q, Kc, Vc, torch.arange(25, **i32)[None], torch.tensor([k], **i32),
                                  torch.tensor([0, new], **i32), max_new=new, scale=1.0)
        assert (O[:, :, 7] == value).all()
        assert O[:, :, :7].isfinite().all() and O[:, :, 8:].isfinite().all()
