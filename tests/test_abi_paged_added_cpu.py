"""Refusals of gs_paged_attention_added and gs_verify_added: the checks run on the
host, so fake addresses reach no kernel."""
import pytest
import torch

from paper_2608_01528_amd import gramspace as gs
from test_abi_paged_cpu import NO_GPU, WS, Attn, Drafts

ADDED = 0x1a000000


@pytest.fixture(scope="module")
def L():
    return gs.lib()


def attend(L, added, n=1 << 30, **change):
    return L.gs_paged_attention_added(Attn(**change).bytes(), added, gs.GS_BF16, WS, n, None)


def verify(L, added, n=1 << 30, **change):
    return L.gs_verify_added(Drafts(**change).bytes(), added, gs.GS_F32, WS, n, None)


@NO_GPU
@pytest.mark.parametrize("call", [attend, verify])
def test_valid_problems_end_with_the_missing_device(L, call):
    assert call(L, ADDED) == gs.GS_ERR_DEVICE and call(L, None) == gs.GS_ERR_DEVICE


@pytest.mark.parametrize("call,added,change,status", [
    (attend, ADDED + 2, {}, gs.GS_ERR_ALIGN), (verify, ADDED + 2, {}, gs.GS_ERR_ALIGN),
    (attend, 0x16000000, {}, gs.GS_ERR_ARG), (attend, 0x17000000, {}, gs.GS_ERR_ARG),       # over O, over lse
    (verify, 0x16000008, {}, gs.GS_ERR_ARG), (verify, 0x17000000, {}, gs.GS_ERR_ARG), (verify, 0x18000010, {}, gs.GS_ERR_ARG),
    (attend, WS, dict(Lk=300, page=64, K=(0x14000000, 8192, 128, 64), V=(0x15000000, 8192, 128, 64)), gs.GS_ERR_ARG),
    (verify, WS, dict(M=50000, ldp=50000, ldq=50000, P=0x20000000, Q=0x30000000), gs.GS_ERR_ARG),
    (attend, ADDED, dict(Lk=81), gs.GS_ERR_SHAPE), (verify, ADDED, dict(M=0), gs.GS_ERR_SHAPE)])
def test_refused(L, call, added, change, status):
    assert call(L, added, **change) == status
    assert L.gs_last_error()


def test_null_problems(L):
    assert L.gs_paged_attention_added(None, ADDED, gs.GS_BF16, WS, 1 << 20, None) == gs.GS_ERR_ARG
    assert L.gs_verify_added(None, ADDED, gs.GS_F32, WS, 1 << 20, None) == gs.GS_ERR_ARG


@pytest.mark.parametrize("change", [dict(B=0), dict(N=0), dict(Lq=0)])
def test_nothing_to_do(L, change):
    assert attend(L, ADDED, **change) == gs.GS_OK
    assert verify(L, ADDED, B=0, N=0) == gs.GS_OK


def test_binding_refuses_host_tensors():
    i = torch.zeros(3, dtype=torch.int32)
    c = torch.zeros(4, 8, 2, 16)
    with pytest.raises(ValueError, match="GPU"):
        gs.gs_paged_attention(torch.zeros(3, 2, 16), c, c, i.view(3, 1), i, added=i)
    with pytest.raises(ValueError, match="GPU"):
        gs.gs_verify(torch.zeros(3, 5), i, torch.zeros(3), torch.zeros(2), i, added=i[:2])
