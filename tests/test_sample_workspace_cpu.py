"""The workspace of gs_sample holds the rows that one round of launches takes,
and no more: 2048, or as many as have 2^22 chunks of 8192 entries."""
import pytest

from paper_2608_01528_amd import gramspace as gs

CHUNK = 8192


def need(B, M, t=gs.GS_BF16):
    return gs.lib().gs_sample_workspace(t, B, M)


@pytest.mark.parametrize("M", [8190, 131072, (1 << 24) - 3, 1 << 24, (1 << 25) + 1, 1 << 28, (1 << 31) - 257])
def test_rows_that_launches_take(M):
    chunks = (M + 3 + CHUNK - 1) // CHUNK
    most = min(2048, (1 << 22) // chunks)
    one = need(1, M)
    assert one > 400 * chunks
    for B in (1, 2, most - 1, most, most + 1, 2048, 5000, 1 << 22):
        if B >= 1:
            assert need(B, M) == min(B, most) * one, B


def test_rows_of_one_work_group_need_none():
    assert need(1 << 22, 8189) == need(5, 22) == 0
