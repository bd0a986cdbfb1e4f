"""A paged cache's operators on the host, from their definitions.

`attention` takes each row's states out of the pages and hands them to
attn_util.reference, whose bounds hold whatever the split over tiles and parts.
The other operators are integers, copies, and draws in 64 bits."""
import numpy as np
import torch

import attn_util


def plan(length, add, table, free, nfree, page, rows):
    """Lists and arrays after a step: (length, nfree, qoff, slots, added, table, free)."""
    up = lambda x: -(-x // page)  # noqa: E731
    B, width = table.shape
    table, free = table.copy(), free.copy()
    most = min(width * page, 2**31 - 1)
    n0 = min(max(nfree, 0), free.size)
    stack = free[:n0].tolist()
    length = [min(max(x, 0), most) for x in length]
    for b in range(B):
        if add[b] < 0:
            left = max(length[b] + add[b], 0)
            stack += table[b, up(left): up(length[b])].tolist()
            length[b] = left
    stack = stack[: free.size]
    free[: len(stack)] = stack
    qoff, slots, added, wanted, avail = [0], np.full(rows, -1, np.int64), [0] * B, 0, len(stack)
    for b in range(B):
        n = max(add[b], 0)
        qoff.append(qoff[-1] + n)
        if n == 0 or length[b] + n > most or qoff[-1] > rows:
            continue
        need = up(length[b] + n) - up(length[b])
        wanted += need
        if need and wanted > avail:
            continue
        for k in range(need):
            table[b, up(length[b]) + k] = stack.pop()
        at = np.arange(length[b], length[b] + n)
        ids = table[b, at // page].astype(np.int64)
        slots[qoff[-2]: qoff[-1]] = np.where(ids < 0, -1, ids * page + at % page)
        length[b] += n
        added[b] = n
    return length, len(stack), [min(x, 2**31 - 1) for x in qoff], slots, added, table, free


def seen(p, klen, window, sinks):
    """States that a row at position p sees."""
    j = np.arange(min(p + 1, klen)) if p >= 0 else np.arange(0)
    return j if window == 0 else j[(j > p - window) | (j < sinks)]


def attention(Q, Kc, Vc, table, klen, qoff, max_new=None, max_len=None, window=0, sinks=0, scale=None):
    """{name: (value, bound)} of O (N, Hq, Dh) and lse (N, Hq), and how many
    requests name each row (a row of two, where offsets fall, holds either's)."""
    Q, Kc, Vc = (t.detach().cpu() for t in (Q, Kc, Vc))
    table, klen = table.cpu().numpy().astype(np.int64), klen.cpu().tolist()
    pages, page = Kc.shape[:2]
    N, Hq, Dh = Q.shape
    room = table.shape[1] * page
    max_len = room if max_len is None else max_len
    off = list(range(N + 1)) if qoff is None else [min(max(x, 0), N) for x in qoff.cpu().tolist()]
    O, lse = torch.zeros(N, Hq, Dh, dtype=torch.float64), torch.zeros(N, Hq, dtype=torch.float64)
    tO, tl = torch.zeros_like(O), torch.zeros_like(lse)
    named = torch.zeros(N, dtype=torch.int32)
    for b, k in enumerate(klen):
        k = min(max(k, 0), max_len)
        n = max(off[b + 1] - off[b], 0)
        for i in range(n if max_new is None else min(n, max_new)):
            r = off[b] + i
            named[r] += 1
            j = seen(k - n + i, k, window, sinks)
            ids = table[b, j // page]
            ok = (ids >= 0) & (ids < pages)
            g, at = torch.from_numpy(ids[ok]), torch.from_numpy((j % page)[ok])
            ref = attn_util.reference(Q[None, r: r + 1], Kc[g, at][None], Vc[g, at][None], scale=scale)
            O[r], tO[r] = ref["O"][0][0, 0], ref["O"][1][0, 0]
            lse[r], tl[r] = ref["lse"][0][0, :, 0], ref["lse"][1][0, :, 0]
    return {"O": (O, tO), "lse": (lse, tl)}, named


def weights(row):
    w = row.astype(np.float64)
    return np.where(np.isfinite(w) & (w > 0), w, 0.0)


def verify(P, Q, drafted, u, v, qoff, near=None):
    """(accepted, entry, entries) on arrays; entries of rows of no request, and of
    rows that two requests name (offsets that fall), are None.
    `near`: a list that gets the relative distance of each draw's target from
    the next border between entries."""
    N, M = P.shape
    clean = lambda x: float(x) if x > 0 else 0.0  # noqa: E731
    off = [min(max(x, 0), N) for x in qoff]
    accepted, entry, entries = [], [], [None] * N
    for b in range(len(v)):
        n = off[b + 1] - off[b]
        if n <= 0:
            accepted.append(0)
            entry.append(-1)
            continue
        a, x = 0, -1
        while a < n - 1:
            r = off[b] + a
            x = int(drafted[r])
            inside = 0 <= x < M
            p = weights(P[r, x: x + 1])[0] if inside else 0.0
            q = (1.0 if Q is None else weights(Q[r, x: x + 1])[0]) if inside else 0.0
            if not clean(u[r]) * q < p:
                break
            entries[r] = x
            a += 1
        r = off[b] + a
        w = p = weights(P[r])
        if a < n - 1:
            q = weights(Q[r]) if Q is not None else (np.arange(M) == x).astype(np.float64)
            w = np.maximum(p - q, 0.0)
            if not w.any():
                w = p
        at = np.nonzero(w)[0]
        e = -1
        if at.size:
            sums = np.cumsum(w[at])
            t = clean(v[b]) * sums[-1]
            k = at.size - 1 if v[b] >= 1 else min(int(np.searchsorted(sums, t, side="right")), at.size - 1)
            e = int(at[k])
            if near is not None and v[b] < 1 and t > 0:
                near.append(float(np.abs(sums[:-1] - t).min() / sums[-1]) if at.size > 1 else 1.0)
        entries[r] = e
        for k in range(a + 1, n):
            entries[off[b] + k] = -1
        accepted.append(a)
        entry.append(e)
    named = np.zeros(N, int)
    for b in range(len(v)):
        named[off[b]: max(off[b], off[b + 1])] += 1
    return accepted, entry, [x if k < 2 else None for x, k in zip(entries, named)]
