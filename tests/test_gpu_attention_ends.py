"""Cross attention at the largest number of states: the last part of a split
sequence ends within 2^31, and what lies in it counts.

All states are 0 but the last n, which are 1, and every query is q: with N = Lk
- n others the last states' probabilities are p1 = e^q / W, the others' p0 = 1 /
W, W = N + n e^q, and

  O = n p1     lse = log W     dQ = O (1 - O)     (dO = 1)
  dK = Lq q p1 (1 - O), -Lq q p0 O     dV = Lq p1, Lq p0

Tolerance: bf16 half steps (2^-8) of the probabilities, of O, of dS and of the
outputs; O's one is as large beside 1 - O, since q makes O about a half; fp32
sums of one part (2^21 steps of whole numbers, or of 2^-21 each) 2^-9 at most."""
import math

import pytest
import torch

from paper_2608_01528_amd import gramspace as gs

pytestmark = pytest.mark.gpu

LK, LAST, Q = 2147482496, 1000, 14.5625     # 2^31 - 1152: (2^24 - 9) blocks of 128


@pytest.fixture(scope="module")
def states():
    K = torch.zeros(1, LK, 1, 1, dtype=torch.bfloat16, device="cuda")
    K[:, -LAST:] = 1.0
    return K


def numbers():
    W = (LK - LAST) + LAST * math.exp(Q)
    return W, math.exp(Q) / W, 1.0 / W


def close(t, want):
    lo, hi = float(t.min()), float(t.max())
    assert abs(lo - want) <= 2.0 ** -5 * abs(want) and abs(hi - want) <= 2.0 ** -5 * abs(want), (lo, hi, want)


@pytest.mark.parametrize("Lq", [1, 33])
def test_the_last_part_counts(states, Lq):
    W, p1, p0 = numbers()
    q = torch.full((1, Lq, 1, 1), Q, dtype=torch.bfloat16, device="cuda")
    O, lse = gs.gs_cross_attention(q, states, states, scale=1.0, lse=True)
    close(O.float(), LAST * p1)
    assert float((lse - math.log(W)).abs().max()) <= 2.0 ** -8


def test_its_gradient(states):
    W, p1, p0 = numbers()
    O = LAST * p1
    Lq = 33
    q = torch.full((1, Lq, 1, 1), Q, dtype=torch.bfloat16, device="cuda")
    o = torch.full_like(q, O)
    lse = torch.full((1, 1, Lq), math.log(W), device="cuda")
    dQ, dK, dV = gs.gs_cross_attention_grad(torch.ones_like(q), q, states, states, o, lse, scale=1.0)
    close(dQ.float(), O * (1 - O))
    close(dV[0, -LAST:].float(), Lq * p1)
    close(dK[0, -LAST:].float(), Lq * Q * p1 * (1 - O))
    close(dV[0, :-LAST], Lq * p0)
    close(dK[0, :-LAST], -Lq * Q * p0 * O)
