"""gs_verify against the definition on the host, in 64 bits.

Products u q and differences p - q of fp32 values are exact in 64 bits up to a
rounding of 2^-53, and a sum of M weights is off by M 2^-53 of the total at
most: draws are compared where the target is further than 4 M 2^-53 of the total
from the border between two entries, which random numbers miss by chance only
(the share of entries within is asserted to be 0)."""
import numpy as np
import pytest
import torch

import paged_util
from paper_2608_01528_amd import gramspace as gs

pytestmark = pytest.mark.gpu
DEV = "cuda"
i32 = torch.int32


def run(P, Q, drafted, u, v, qoff, **kw):
    t = lambda x, dt: torch.as_tensor(np.asarray(x), dtype=dt, device=DEV)  # noqa: E731
    return gs.gs_verify(P, t(drafted, i32), t(u, torch.float32), t(v, torch.float32), t(qoff, i32), Q=Q, entries=True, **kw)


def check(P, Q, drafted, u, v, qoff, **kw):
    near = []
    host = lambda x: None if x is None else x.float().cpu().numpy()  # noqa: E731
    u, v = np.asarray(u, np.float32), np.asarray(v, np.float32)
    want = paged_util.verify(host(P), host(Q), drafted, u, v, qoff, near)
    assert all(x > 4 * P.shape[1] * 2.0**-53 for x in near)
    acc, entry, entries = run(P, Q, drafted, u, v, qoff, **kw)
    assert acc.tolist() == want[0]
    assert entry.tolist() == want[1]
    for g, w in zip(entries.tolist(), want[2]):
        assert w is None or g == w
    return want


def case(seed, B, M, most, dtype, draft, ld=None):
    rng = np.random.default_rng(seed)
    n = rng.integers(0, most + 2, B)
    qoff = np.concatenate([[0], np.cumsum(n)])
    N = int(qoff[-1])
    x = rng.normal(size=(N, M)) * 2.5
    y = x + 0.6 * rng.normal(size=(N, M))
    x[(x < 0) & (x < x.max(1, keepdims=True, initial=-99))] = -np.inf
    soft = lambda z: np.exp(z - z.max(1, keepdims=True)) / np.exp(z - z.max(1, keepdims=True)).sum(1, keepdims=True)  # noqa: E731
    p, q = soft(x) if N else x, soft(y) if N else y
    drafted = (q / rng.exponential(size=q.shape)).argmax(1) if N else np.zeros(0, int)

    def put(z):
        t = torch.full((N, ld or M), float("nan"), dtype=dtype, device=DEV)
        t[:, :M] = torch.from_numpy(z).to(DEV).to(dtype)
        return t[:, :M]

    return put(p), put(q) if draft else None, drafted, rng.random(N).astype(np.float32), rng.random(B).astype(np.float32), qoff


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,M,most", [(1, 1, 1), (3, 2, 2), (50, 22, 4), (20, 1000, 5), (9, 4096, 3), (9, 4097, 3),
                                      (5, 12289, 4), (2, 131072, 2)])
def test_verify(B, M, most, dtype, draft):
    check(*case(B + M, B, M, most, dtype, draft))


def test_long_runs_of_drafts():
    """Runs of more drafts than a wave has lanes, taken to every length."""
    M, n = 7, 200
    ends = [0, 1, 63, 64, 65, 127, 128, 198, 199]
    rng = np.random.default_rng(4)
    P = torch.rand(n * len(ends), M, device=DEV) + 0.5
    drafted = rng.integers(0, M, n * len(ends))
    u = np.zeros(n * len(ends))
    for k, e in enumerate(ends):
        if e < n - 1:
            u[k * n + e] = 2.0          # q u above any p
    qoff = np.arange(len(ends) + 1) * n
    want = check(P, None, drafted, u, rng.random(len(ends)), qoff)
    assert want[0] == [min(e, n - 1) for e in ends]


@pytest.mark.parametrize("M", [50, 9000])
def test_draws_at_the_ends(M):
    """Random numbers at 0, below, at 1, above and NaN; rows of a single weight."""
    P = torch.zeros(6, M, device=DEV)
    P[:, [3, M - 5]] = 0.5
    P[4] = 0
    P[4, M - 1] = 1e-30
    P[5] = 0
    v = np.array([0.0, -1.0, 1.0, float("nan"), 0.7, 0.3], np.float32)
    acc, entry, _ = run(P, None, [0] * 6, [0.5] * 6, v, list(range(7)))
    assert acc.tolist() == [0] * 6 and entry.tolist() == [3, 3, M - 5, 3, M - 1, -1]
    assert run(P, None, [0] * 6, [0.5] * 6, np.full(6, np.inf, np.float32), list(range(7)))[1].tolist() == [M - 5] * 4 + [M - 1, -1]


@pytest.mark.parametrize("M", [40, 5000])
def test_nothing_left_of_the_difference(M):
    """Where q covers p the entry is drawn from p; where p has nothing either, none."""
    P = torch.zeros(6, M, device=DEV)
    P[0::2, 5], P[0::2, M - 2] = 0.25, 0.75
    Q = P + 0.1
    P[4] = 0
    for v, e in ((0.1, 5), (0.3, M - 2)):
        acc, entry, _ = run(P, Q, [5] * 6, [1.0] * 6, [v] * 3, [0, 2, 4, 6])
        assert acc.tolist() == [0, 0, 0] and entry.tolist() == [e, e, -1]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M", [64, 4200])
def test_values_without_weight(M, dtype):
    """Negative, infinite and NaN probabilities count as 0, in drafts, differences and draws."""
    g = np.random.default_rng(M)
    P, Q, drafted, u, v, qoff = case(M, 12, M, 3, dtype, True)
    for t in (P, Q):
        for value in (float("nan"), float("inf"), -float("inf"), -0.5):
            at = torch.from_numpy(g.random(tuple(t.shape)) < 0.1).to(DEV)
            t.masked_fill_(at, value)
    u[::3], v[::5] = float("nan"), -2.0
    check(P, Q, drafted, u, v, qoff)


def test_drafts_outside_the_table_and_rows_out_of_range():
    P, Q, drafted, u, v, qoff = case(8, 10, 33, 3, torch.float32, True)
    drafted[::2] = np.resize([-1, 33, 2**31 - 1, -2**31], drafted[::2].size)
    check(P, Q, drafted, u, v, qoff)
    check(P, None, drafted, u, v, qoff)
    # offsets beyond the rows, falling ones: clamped, a request without rows
    N = P.shape[0]
    check(P, Q, drafted, u, v[:4], [-5, 3, 2, N + 9, N + 9])


@pytest.mark.parametrize("ld", [41, 48, 5001, 5008])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_inside_wider_ones(ld, dtype):
    M = ld - 1 if ld < 100 else 5000
    check(*case(ld, 7, M, 3, dtype, True, ld=ld))


def test_first_address_off_its_boundary():
    P, Q, drafted, u, v, qoff = case(3, 6, 5001, 2, torch.float32, True)
    check(P[:, 1:], Q[:, 3:4] * 0 + Q[:, 1:], np.minimum(drafted, 4999), u, v, qoff)


def test_rows_of_no_request_are_left():
    P, Q, drafted, u, v, _ = case(5, 6, 30, 3, torch.float32, True)
    N = P.shape[0]
    given = torch.full((N,), 77, dtype=i32, device=DEV)
    run(P, Q, drafted, u, v[:2], [1, 3, N - 1], entries_out=given)
    assert given[0] == 77 and given[N - 1] == 77 and (given[1: N - 1] != 77).all()


def test_captured_and_at_once_on_two_streams():
    a, b = case(1, 4, 9000, 3, torch.float32, True), case(2, 4, 9000, 3, torch.float32, True)
    t = lambda x, dt: torch.as_tensor(np.asarray(x), dtype=dt, device=DEV)  # noqa: E731
    ready = [(c[0], t(c[2], i32), t(c[3], torch.float32), t(c[4], torch.float32), t(c[5], i32), c[1]) for c in (a, b)]
    want = [tuple(x.clone() for x in gs.gs_verify(*r, entries=True)) for r in ready]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ready]
    for _ in range(5):
        got = []
        for s, r in zip(streams, ready):
            with torch.cuda.stream(s):
                got.append(gs.gs_verify(*r, entries=True))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for w, o in zip(want, got) for x, y in zip(w, o))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = gs.gs_verify(*ready[0], entries=True)
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want[0]))


def test_far_rows():
    """Probabilities more than 2^31 values from the first."""
    M, N = 131072, 20000
    if torch.cuda.mem_get_info()[0] < 2 * N * M * 2:
        pytest.skip("not enough memory")
    P = torch.zeros(N, M, dtype=torch.bfloat16, device=DEV)
    P[N - 2, 77], P[N - 2, 90000], P[N - 1, 131071] = 0.5, 0.5, 1.0
    u, drafted = torch.zeros(N, device=DEV), torch.full((N,), 90000, dtype=i32, device=DEV)
    q = torch.tensor([N - 2, N], dtype=i32, device=DEV)
    acc, entry, entries = gs.gs_verify(P, drafted, u, torch.tensor([0.4], device=DEV), q, entries=True)
    assert acc.tolist() == [1] and entry.tolist() == [131071] and entries[N - 2:].tolist() == [90000, 131071]
