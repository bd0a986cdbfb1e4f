"""Arguments of the sequence operators' binding: outputs that are given are
written, numbers beyond fp32 are taken as infinite, heads of no values are
refused by the library."""
import pytest
import torch

from paper_2608_01528_amd import gramspace as gs

pytestmark = pytest.mark.gpu


def test_outputs_that_are_given_are_written():
    S, u = torch.randn(9, 70, device="cuda"), torch.rand(9, device="cuda")
    idx, prob, kept = gs.gs_sample(S, u, top_k=5, prob=True, kept=True)
    p, k = torch.full((9,), 7.0, device="cuda"), torch.full((9,), 7, dtype=torch.int32, device="cuda")
    got = gs.gs_sample(S, u, top_k=5, prob_out=p, kept_out=k)
    assert isinstance(got, torch.Tensor) and torch.equal(got, idx)
    assert torch.equal(p, prob) and torch.equal(k, kept)
    p.fill_(7.0)
    got = gs.gs_sample(S, u, top_k=5, kept=True, prob_out=p)
    assert len(got) == 2 and torch.equal(got[1], kept) and torch.equal(p, prob)
    with pytest.raises(ValueError, match="prob_out"):
        gs.gs_sample(S, u, prob_out=p[:5])
    Q, K = torch.randn(2, 3, 2, 64, device="cuda"), torch.randn(2, 5, 1, 64, device="cuda")
    O, lse = gs.gs_cross_attention(Q, K, K, lse=True)
    stats = torch.zeros_like(lse)
    assert torch.equal(gs.gs_cross_attention(Q, K, K, lse_out=stats), O) and torch.equal(stats, lse)


def test_numbers_beyond_fp32():
    S, u = torch.randn(6, 40, device="cuda"), torch.rand(6, device="cuda")
    inf = float("inf")
    for far, near in (({"temperature": 1e300}, {"temperature": inf}), ({"temperature": -1e300}, {"temperature": 0.0}),
                      ({"top_p": 1e200}, {}), ({"min_p": 1e39}, {"min_p": 1.0}), ({"top_k": 1 << 40}, {}), ({"temperature": 2}, {"temperature": 2.0})):
        for a, b in zip(gs.gs_sample(S, u, prob=True, kept=True, **far), gs.gs_sample(S, u, prob=True, kept=True, **near)):
            assert torch.equal(a, b), far


def test_heads_of_no_values_are_refused():
    Q, K = torch.empty(2, 3, 2, 0, device="cuda"), torch.empty(2, 5, 1, 0, device="cuda")
    with pytest.raises(gs.GramSpaceError, match="Dh"):
        gs.gs_cross_attention(Q, K, K)
    with pytest.raises(gs.GramSpaceError, match="Dh"):
        gs.gs_cross_attention_grad(Q, Q, K, K, Q, torch.empty(2, 2, 3, device="cuda"))
