"""One step of serving from a paged cache: pages dealt out, states stored, attention over them, drafted entries verified.

Each case is one call of the step that a program repeats while it answers
requests.  The states (keys and values) of all requests lie in pages of one
cache; `plan` gives each request the pages and slots of its new positions,
`store` writes their states there, `attend` is the new positions' attention
over all that their request has in the cache, and `verify` takes or refuses the
entries that a smaller model drafted, by the probabilities at those positions.

`own` chooses between the operators' plain forms, written with elementary torch
operations (`attend` in 32 bits; `verify` in 64: entries are taken and drawn by
comparing products and sums with random numbers), and the library's calls.
`exact` computes the same outputs from the definitions in 64 bits.

Sizes.  B requests; pages of `page` positions; Hkv heads of Dh values.
attend: up to `new` new positions a request (`ragged`: fewer in most, none in
the last of three or more) at the end of up to Lk states, Hq query heads over
Hkv; `window` > 0: a position sees the last `window` states and the first
`sinks`.  verify: up to `new` drafted entries a request out of M; `draft`: their
own probabilities are given.
"""
import math

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda"


# ------------------------------------------------------------------ cases

def listed():
    return [
        # a decoding step's bookkeeping: one more position for most requests, some ended, some taking drafts back
        {"name": "plan_step", "kind": "plan", "B": 250, "page": 16, "width": 500, "new": 4, "prompts": False},
        # a wave of prompts arrives: long runs of new slots
        {"name": "plan_prompts", "kind": "plan", "B": 700, "page": 32, "width": 256, "new": 2000, "prompts": True},
        # the states of one decoding step of a full batch
        {"name": "store_step", "kind": "store", "dtype": "bf16", "cache": "bf16", "N": 190, "page": 16, "pages": 1500,
         "Hkv": 8, "Dh": 128},
        # the states of whole prompts, computed in fp32, kept in bf16
        {"name": "store_prompts", "kind": "store", "dtype": "f32", "cache": "bf16", "N": 16000, "page": 32,
         "pages": 600, "Hkv": 8, "Dh": 128},
        # one new token of four requests with short histories: latency
        {"name": "token_short", "kind": "attend", "dtype": "bf16", "B": 4, "new": 1, "Lk": 77, "page": 16, "Hq": 8,
         "Hkv": 8, "Dh": 64, "ragged": True, "window": 0, "sinks": 0},
        # one new token of each request of a serving batch, histories of all lengths
        {"name": "token_batch", "kind": "attend", "dtype": "bf16", "B": 48, "new": 1, "Lk": 7000, "page": 16, "Hq": 32,
         "Hkv": 8, "Dh": 128, "ragged": True, "window": 0, "sinks": 0},
        # one request's very long history: the axis of the states is all there is to share out
        {"name": "token_long", "kind": "attend", "dtype": "bf16", "B": 1, "new": 1, "Lk": 200001, "page": 64, "Hq": 32,
         "Hkv": 4, "Dh": 128, "ragged": False, "window": 0, "sinks": 0},
        # drafted tokens (and the one before them) verified at once, fp32, a window with sinks, pages that end inside tiles
        {"name": "drafts_window_fp32", "kind": "attend", "dtype": "f32", "B": 40, "new": 5, "Lk": 6000, "page": 24,
         "Hq": 16, "Hkv": 8, "Dh": 80, "ragged": True, "window": 2000, "sinks": 4},
        # pieces of prompts on top of what is in the cache already
        {"name": "prompt_pieces", "kind": "attend", "dtype": "bf16", "B": 5, "new": 1500, "Lk": 6000, "page": 16,
         "Hq": 32, "Hkv": 8, "Dh": 128, "ragged": True, "window": 0, "sinks": 0},
        # one request's drafted entries out of a language-sized table: latency
        {"name": "verify_one", "kind": "verify", "dtype": "f32", "B": 1, "new": 4, "M": 131072, "draft": True},
        # a serving batch, probabilities in bf16
        {"name": "verify_batch", "kind": "verify", "dtype": "bf16", "B": 120, "new": 5, "M": 50257, "draft": True},
        # drafts found by lookup (no probabilities of their own) out of a compressed codebook
        {"name": "verify_codebook", "kind": "verify", "dtype": "f32", "B": 2000, "new": 3, "M": 1843, "draft": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "store", "attend", "attend", "attend", "verify", "verify"])
    page = rng.choice([1, 8, 16, 16, 24, 32, 64, 100, 128])
    if kind == "plan":
        prompts = rng.random() < 0.5
        B = _log(rng, 1, 4000)
        new = _log(rng, 2, max(3, min(4000, 1400000 // B))) if prompts else rng.choice([1, 1, 3, 8])
        width = max(2, min(_log(rng, 64, 8192) // page + 1, (1 << 21) // B))
        return {"kind": kind, "B": B, "page": page, "width": width, "new": new, "prompts": prompts}
    if kind == "store":
        Hkv, Dh = rng.choice([1, 2, 4, 8]), rng.choice([32, 40, 64, 72, 96, 128])
        N = _log(rng, 1, min(16000, (1 << 24) // (Hkv * Dh)))
        return {"kind": kind, "dtype": rng.choice(["bf16", "f32"]), "cache": rng.choice(["bf16", "bf16", "f32"]), "N": N,
                "page": page, "pages": N // page + 1 + _log(rng, 1, 300), "Hkv": Hkv, "Dh": Dh}
    if kind == "verify":
        M = _log(rng, 2, 131072)
        new = rng.choice([0, 1, 2, 4, 5, 8])
        return {"kind": kind, "dtype": rng.choice(["f32", "bf16"]), "new": new, "M": M,
                "B": _log(rng, 1, max(1, min(2000, (1 << 25) // (M * (new + 1))))), "draft": rng.random() < 0.7}
    dtype = rng.choice(["bf16", "bf16", "f32"])
    Dh = rng.choice([32, 40, 64, 64, 80, 96, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    Hq = Hkv * rng.choice([1, 1, 2, 4, 5, 8])
    what = rng.choice(["token", "token", "drafts", "prompt"])
    if what == "prompt":
        new, Lk = _log(rng, 9, 2000), _log(rng, 40, 8192)
    else:
        new, Lk = (1 if what == "token" else rng.choice([2, 3, 5, 8])), _log(rng, 8, 65536)
    Lk = max(Lk, new)
    pairs = 1 << (30 if dtype == "bf16" else 27)        # B Hq new Lk
    B = _log(rng, 1, max(1, min(128, pairs // (Hq * new * Lk), (1 << 27) // (Hkv * Lk * Dh))))
    window = 0 if rng.random() < 0.6 else _log(rng, 8, max(9, Lk))
    return {"kind": kind, "dtype": dtype, "B": B, "new": new, "Lk": Lk, "page": page, "Hq": Hq, "Hkv": Hkv, "Dh": Dh,
            "ragged": rng.random() < 0.6, "window": window, "sinks": rng.choice([0, 1, 4, 20]) if window else 0}


def lengths(c):
    """New positions and states of each request of an `attend` case (a case's own, whatever the seed)."""
    B, new, Lk = c["B"], c["new"], c["Lk"]
    if not c["ragged"]:
        return [new] * B, [Lk] * B
    n = [new - (13 * b) % new for b in range(B)]
    k = [max(Lk - (997 * b) % Lk, n[b]) for b in range(B)]
    if B > 2 and new > 1:
        n[B - 1] = 0
    return n, k


def _rows(c):
    """Rows that a step has room for: a little more than a `plan` case's requests ask for as a rule."""
    return c["B"] * (c["new"] + 1) // 2 + c["new"] if c["prompts"] else 2 * c["B"] + c["new"]


def _seen(c, n, k):
    """States that some row of a request sees, and (row, state) pairs."""
    if not c["window"]:
        return k if n else 0, n * k - n * (n - 1) // 2
    w, s = c["window"], c["sinks"]
    first = max(0, k - n - w + 1)
    pos = np.arange(k - n, k, dtype=np.int64)
    lo = np.maximum(0, pos - w + 1)
    return (k - first + min(s, first)) if n else 0, int((pos + 1 - lo + np.minimum(s, lo)).sum())


def work(c):
    if c["kind"] == "plan":     # per request lengths read and written; per new position a slot written; a page each P
        rows = _rows(c)
        return {"bytes": 24 * c["B"] + 8 * rows + 8 * (rows // c["page"] + c["B"] // 8), "flops": 4 * rows + 10 * c["B"]}
    if c["kind"] == "store":
        e = (2 if c["dtype"] == "bf16" else 4) + (2 if c["cache"] == "bf16" else 4)
        return {"bytes": c["N"] * (2 * c["Hkv"] * c["Dh"] * e + 8), "flops": 0}
    if c["kind"] == "verify":   # the row that is drawn from, of both; the drafts' entries; per entry a difference and a sum
        e = 2 if c["dtype"] == "bf16" else 4
        rows = 2 if c["draft"] else 1
        return {"bytes": c["B"] * (rows * c["M"] * e + c["new"] * 3 * 4 + 24), "flops": 2 * c["B"] * c["M"]}
    e = 2 if c["dtype"] == "bf16" else 4
    n, k = lengths(c)
    seen = [_seen(c, a, b) for a, b in zip(n, k)]
    states, pairs, rows = sum(x for x, _ in seen), sum(x for _, x in seen), sum(n)
    by = e * c["Dh"] * (2 * states * c["Hkv"] + 2 * rows * c["Hq"]) + 4 * rows * c["Hq"] + 4 * states // c["page"]
    return {"bytes": by, "flops": 4 * pairs * c["Hq"] * c["Dh"]}


# ------------------------------------------------------------------ inputs

def prepare(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"case": dict(c)}
    return {"plan": _prepare_plan, "store": _prepare_store, "attend": _prepare_attend,
            "verify": _prepare_verify}[c["kind"]](c, s, g)


def _int(x):
    return x.to(torch.int32)


def _prepare_plan(c, s, g):
    B, page, width, new = c["B"], c["page"], c["width"], c["new"]
    room = page * width
    uni = lambda lo, hi: torch.randint(lo, hi + 1, (B,), generator=g, device=DEV)  # noqa: E731
    if c["prompts"]:    # most requests are new, some of the prompts are longer than a table has room for
        length = torch.where(uni(0, 3) == 0, uni(0, room), 0)
        add = uni(1, new)
    else:               # one more, now and then a run of accepted drafts; drafts taken back; requests that ended
        length = uni(0, room)
        kind = uni(0, 19)
        add = torch.where(kind < 15, 1, torch.where(kind < 17, uni(1, new), torch.where(kind < 19, -uni(0, new), -length)))
    held = (length + page - 1) // page
    wanted = (length + add.clamp(min=0) + page - 1) // page - held
    total, most = int(held.sum()), B * width + 2
    nfree = min(int(0.97 * wanted.sum()) + 2, most - total)     # a few requests find too few
    order = torch.randperm(most, generator=g, device=DEV, dtype=torch.int32)
    at = held.cumsum(0) - held
    col = torch.arange(width, device=DEV)[None, :]
    s["table"] = torch.where(col < held[:, None], order[(at[:, None] + col).clamp(max=most - 1)], -1)
    s["free"] = torch.full((most,), -1, device=DEV, dtype=torch.int32)
    s["free"][:nfree] = order[total: total + nfree]
    s["nfree"] = torch.tensor([nfree], device=DEV, dtype=torch.int32)
    s["length"], s["add"], s["rows"] = _int(length), _int(add), _rows(c)
    return s


def _prepare_store(c, s, g):
    N, page, pages, Hkv, Dh = (c[k] for k in ("N", "page", "pages", "Hkv", "Dh"))
    normal = lambda *n: torch.randn(*n, generator=g, device=DEV)  # noqa: E731
    s["K"], s["V"] = normal(N, Hkv, Dh).to(DT[c["dtype"]]), normal(N, Hkv, Dh).to(DT[c["dtype"]])
    s["Kc"], s["Vc"] = (normal(pages, page, Hkv, Dh).to(DT[c["cache"]]) for _ in range(2))
    # runs of slots, a page each, in pages from anywhere; padding rows at the end
    order = torch.randperm(pages, generator=g, device=DEV)
    i = torch.arange(N, device=DEV)
    s["slots"] = order[i // page] * page + i % page
    s["slots"][N - N // 16:] = -1
    return s


def _prepare_attend(c, s, g):
    B, page, Hq, Hkv, Dh = (c[k] for k in ("B", "page", "Hq", "Hkv", "Dh"))
    n, k = lengths(c)
    dt = DT[c["dtype"]]
    held = [-(-x // page) for x in k]
    pages = sum(held) + 3
    normal = lambda *m: torch.randn(*m, generator=g, device=DEV, dtype=dt)  # noqa: E731
    s["Kc"], s["Vc"] = normal(pages, page, Hkv, Dh), normal(pages, page, Hkv, Dh)
    s["Q"] = normal(sum(n), Hq, Dh)
    order = torch.randperm(pages, generator=g, device=DEV, dtype=torch.int32)
    h = torch.tensor(held, device=DEV)
    col = torch.arange(max(held), device=DEV)[None, :]
    s["table"] = torch.where(col < h[:, None], order[((h.cumsum(0) - h)[:, None] + col).clamp(max=pages - 1)], -1)
    s["klen"] = torch.tensor(k, device=DEV, dtype=torch.int32)
    s["qoff"] = torch.tensor([0] + list(np.cumsum(n)), device=DEV, dtype=torch.int32)
    s["max_new"], s["max_len"], s["scale"] = max(n), max(k), 1.0 / math.sqrt(Dh)
    return s


def _prepare_verify(c, s, g):
    B, M, new = c["B"], c["M"], c["new"]
    n = [1 + (new if b % 3 else new - b % (new + 1)) for b in range(B)]        # rows: the drafts and one more
    N = sum(n)
    x = torch.randn(N, M, generator=g, device=DEV) * 2.5
    y = x + 0.8 * torch.randn(N, M, generator=g, device=DEV)                   # the drafting model's scores
    x.masked_fill_((x < 0) & (x < x.amax(1, keepdim=True)), -math.inf)         # the tail, left out by top_p
    s["P"] = torch.softmax(x, 1).to(DT[c["dtype"]])
    q = torch.softmax(y, 1)
    e = torch.empty(N, M, device=DEV).exponential_(generator=g)
    s["drafted"] = _int((q / e).argmax(1))                                     # drawn from q
    s["Q"] = q.to(DT[c["dtype"]]) if c["draft"] else None
    s["u"] = torch.rand(N, generator=g, device=DEV)
    s["v"] = torch.rand(B, generator=g, device=DEV)
    s["qoff"] = torch.tensor([0] + list(np.cumsum(n)), device=DEV, dtype=torch.int32)
    s["max_new"] = max(n)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _run_own(s)
    return {"plan": _plain_plan, "store": _plain_store, "attend": _plain_attend,
            "verify": _plain_verify}[s["case"]["kind"]](s)


def _run_own(s):
    from paper_2608_01528_amd import gramspace as gs

    c = s["case"]
    if c["kind"] == "plan":
        length, nfree, qoff, slots, added = gs.gs_paged_plan(s["length"], s["add"], s["table"], s["free"], s["nfree"],
                                                             page=c["page"], rows=s["rows"])
        return {"length": length, "nfree": nfree, "qoff": qoff, "slots": slots, "added": added, "table": s["table"],
                "free": s["free"]}
    if c["kind"] == "store":
        gs.gs_paged_store(s["K"], s["V"], s["slots"], s["Kc"], s["Vc"])
        return {"Kc": s["Kc"], "Vc": s["Vc"]}
    if c["kind"] == "verify":
        accepted, entry, entries = gs.gs_verify(s["P"], s["drafted"], s["u"], s["v"], s["qoff"], Q=s["Q"],
                                                entries=True)
        return {"accepted": accepted, "entry": entry, "entries": entries}
    O, lse = gs.gs_paged_attention(s["Q"], s["Kc"], s["Vc"], s["table"], s["klen"], qoff=s["qoff"],
                                   max_new=s["max_new"], max_len=s["max_len"], window=c["window"], sinks=c["sinks"],
                                   scale=s["scale"], lse=True)
    return {"O": O, "lse": lse}


def _plain_plan(s):
    """Requests in order.  A negative `add` takes positions back and returns the pages behind them to the end of the
    free list; then pages are taken from its end, until a request finds too few (that one and later ones that need
    pages get nothing, and so do requests whose table or rows have no room).  Slots are page * P + place in the page;
    rows of requests that got nothing, and rows behind the last one, are -1."""
    page, table, free, rows = s["case"]["page"], s["table"], s["free"], s["rows"]
    B, width = table.shape
    dev = table.device
    length, add = s["length"].long(), s["add"].long()
    n, left = add.clamp(min=0), (length + add.clamp(max=0)).clamp(min=0)
    ends = n.cumsum(0)
    held, stay, want = ((x + page - 1) // page for x in (length, left, left + n))
    back = held - stay
    fits = (want <= width) & (ends <= rows)
    need = torch.where(fits, want - stay, 0) * (add > 0)
    nfree = s["nfree"].long()
    avail = nfree + back.sum()
    taken = need.cumsum(0)
    served = fits & ((need == 0) | (taken <= avail)) & (add > 0)
    need = need * served
    col = torch.arange(width, device=dev)[None, :]
    # pages given back, in order, behind the free ones
    gone = (col >= stay[:, None]) & (col < held[:, None])
    place = nfree + (back.cumsum(0) - back)[:, None] + col - stay[:, None]
    free[place[gone]] = table[gone]
    # pages taken, from the end
    fresh = (col >= stay[:, None]) & (col < (stay + need)[:, None])
    place = avail - 1 - ((need.cumsum(0) - need)[:, None] + col - stay[:, None])
    table[fresh] = free[place[fresh]]
    got = torch.where(served, n, 0)
    r = torch.arange(rows, device=dev)
    b = torch.searchsorted(ends, r, right=True).clamp(max=B - 1)
    at = left[b] + r - (ends - n)[b]
    slots = table[b, (at // page).clamp(max=width - 1)].long() * page + at % page
    slots = torch.where((r < ends[-1]) & served[b], slots, -1)
    qoff = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), ends])
    return {"length": _int(left + got), "nfree": _int(avail - need.sum()), "qoff": _int(qoff), "slots": slots,
            "added": _int(got), "table": table, "free": free}


def _plain_store(s):
    """Row n of K and V to slot slots[n] of the cache, rounded to the cache's type; rows without a slot nowhere."""
    there = s["slots"] >= 0
    at = s["slots"][there]
    s["Kc"].view(-1, *s["Kc"].shape[2:])[at] = s["K"][there].to(s["Kc"].dtype)
    s["Vc"].view(-1, *s["Vc"].shape[2:])[at] = s["V"][there].to(s["Vc"].dtype)
    return {"Kc": s["Kc"], "Vc": s["Vc"]}


def _plain_attend(s):
    """O = softmax(scale Q K^T) V in fp32, the states of all requests brought out of their pages first.  Row i of a
    request's n stands at position p = klen - n + i and sees the states j <= p with j > p - window or j < sinks."""
    c = s["case"]
    B, page, Hq, Hkv, Dh, Lq, Lk = c["B"], c["page"], c["Hq"], c["Hkv"], c["Dh"], s["max_new"], s["max_len"]
    G, dev, dt = Hq // Hkv, s["Q"].device, s["Q"].dtype
    j = torch.arange(Lk, device=dev)
    live = j[None, :] < s["klen"][:, None]
    slot = torch.where(live, s["table"].long()[:, j // page] * page + j % page, 0)

    def states(cache):
        t = cache.view(-1, Hkv, Dh)[slot].float()
        return t.mul_(live[:, :, None, None]).permute(0, 2, 1, 3).reshape(B * Hkv, Lk, Dh)

    first, n = s["qoff"][:-1].long(), (s["qoff"][1:] - s["qoff"][:-1]).long()
    i = torch.arange(Lq, device=dev)
    there = i[None, :] < n[:, None]
    r = torch.where(there, first[:, None] + i[None, :], 0)
    q = s["Q"][r].float().view(B, Lq, Hkv, G, Dh).permute(0, 2, 3, 1, 4).reshape(B * Hkv, G * Lq, Dh)
    p = (s["klen"].long() - n)[:, None] + i[None, :]
    sees = live[:, None, :] & (j[None, None, :] <= p[:, :, None])
    if c["window"]:
        sees &= (j[None, None, :] > p[:, :, None] - c["window"]) | (j < c["sinks"])[None, None, :]
    x = torch.matmul(q, states(s["Kc"]).transpose(1, 2)).mul_(s["scale"]).view(B, Hkv, G, Lq, Lk)
    x.masked_fill_(~sees[:, None, None], -math.inf)
    m = x.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    x.sub_(m).exp_()
    l = x.sum(dim=-1, keepdim=True)
    lse = (m + l.log()).view(B, Hq, Lq).transpose(1, 2)
    x.div_(torch.where(l == 0, 1.0, l))
    o = torch.matmul(x.view(B * Hkv, G * Lq, Lk), states(s["Vc"]))
    o = o.view(B, Hkv, G, Lq, Dh).permute(0, 3, 1, 2, 4).reshape(B, Lq, Hq, Dh)
    return {"O": o[there].to(dt), "lse": lse[there].contiguous()}


def _plain_verify(s):
    """A request's rows: one for each draft and one more.  Draft x of row i is taken if u q(x) < p(x) and all before
    it were; the entry after the last one taken is drawn from max(p - q, 0) of the first row not taken, from p of the
    last row if all were (and where max(p - q, 0) is nothing).  Without Q a draft has q = 1 at its entry."""
    P, Q, u, v, drafted = s["P"], s["Q"], s["u"].double(), s["v"].double(), s["drafted"].long()
    N, M = P.shape
    dev = P.device
    first, n = s["qoff"][:-1].long(), (s["qoff"][1:] - s["qoff"][:-1]).long()
    r = torch.arange(N, device=dev)
    p = P[r, drafted].double()
    q = Q[r, drafted].double() if Q is not None else torch.ones_like(p)
    ok = u * q < p
    i = torch.arange(s["max_new"], device=dev)
    row = (first[:, None] + i[None, :]).clamp(max=N - 1)
    run_ = (ok[row] & (i[None, :] < (n - 1)[:, None])).long().cumprod(1)
    a = run_.sum(1)
    at = (first + a).clamp(max=N - 1)
    w = P[at].double()
    full = w
    less = Q[at].double() if Q is not None else (torch.arange(M, device=dev)[None, :] == drafted[at][:, None]).double()
    w = torch.where((a < n - 1)[:, None], (w - less).clamp_(min=0.0), w)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, full)
    c = w.cumsum(1)
    hit = (c > v[:, None] * c[:, -1:]) & (w > 0)
    e = torch.where(hit, torch.arange(M, device=dev)[None, :], M).amin(1)
    e = torch.where(e == M, -1, e)
    b = torch.searchsorted(s["qoff"][1:].long(), r, right=True)
    k = r - first[b]
    entries = torch.where(k < a[b], drafted, torch.where(k == a[b], e[b], -1))
    return {"accepted": _int(a), "entry": _int(e), "entries": _int(entries)}


# ------------------------------------------------------------------ 64 bits, from the definitions

def exact(c, seed):
    s = prepare(c, seed)
    return {"plan": _exact_plan, "store": _exact_store, "attend": _exact_attend,
            "verify": _exact_verify}[c["kind"]](s, c)


def _exact_plan(s, c):
    """Request by request on the host, the free pages as a list."""
    page, rows = c["page"], s["rows"]
    table, free = s["table"].cpu().numpy().copy(), s["free"].cpu().numpy().copy()
    length, add = s["length"].cpu().tolist(), s["add"].cpu().tolist()
    B, width = table.shape
    stack = free[: int(s["nfree"])].tolist()
    up = lambda x: -(-x // page)  # noqa: E731
    for b in range(B):
        if add[b] < 0:
            left = max(0, length[b] + add[b])
            stack += table[b, up(left): up(length[b])].tolist()
            length[b] = left
    free[: len(stack)] = stack
    qoff, slots, added, wanted, avail = [0], np.full(rows, -1, np.int64), [0] * B, 0, len(stack)
    for b in range(B):
        n = max(0, add[b])
        qoff.append(qoff[-1] + n)
        if n == 0 or up(length[b] + n) > width or qoff[-1] > rows:
            continue
        need = up(length[b] + n) - up(length[b])
        wanted += need
        if need and wanted > avail:
            continue
        for k in range(need):
            table[b, up(length[b]) + k] = stack.pop()
        at = np.arange(length[b], length[b] + n)
        slots[qoff[-2]: qoff[-1]] = table[b, at // page].astype(np.int64) * page + at % page
        length[b] += n
        added[b] = n
    i32 = lambda x: np.asarray(x, np.int32)  # noqa: E731
    return {"length": i32(length), "nfree": i32([len(stack)]), "qoff": i32(qoff), "slots": slots, "added": i32(added),
            "table": table, "free": free}


def _exact_store(s, c):
    slots = s["slots"].cpu().numpy()
    rows = np.nonzero(slots >= 0)[0]
    out = {}
    for cache, x in (("Kc", "K"), ("Vc", "V")):
        t = s[cache].double()
        where = torch.from_numpy(slots[rows]).to(DEV)
        t.view(-1, c["Hkv"], c["Dh"]).index_copy_(0, where, s[x].double()[torch.from_numpy(rows).to(DEV)])
        out[cache] = t
    return out


def _exact_attend(s, c):
    """Request by request and head by head over the states that a request has."""
    B, page, Hq, Hkv, Dh = (c[k] for k in ("B", "page", "Hq", "Hkv", "Dh"))
    n, k = lengths(c)
    G = Hq // Hkv
    f64 = dict(dtype=torch.float64, device=DEV)
    O, lse = torch.zeros(sum(n), Hq, Dh, **f64), torch.zeros(sum(n), Hq, **f64)
    Kc, Vc = s["Kc"].view(-1, Hkv, Dh), s["Vc"].view(-1, Hkv, Dh)
    table, r0 = s["table"].cpu().numpy().astype(np.int64), 0
    for b in range(B):
        at = np.arange(k[b])
        at = torch.from_numpy(table[b, at // page] * page + at % page).to(DEV)
        pos = torch.arange(k[b] - n[b], k[b], device=DEV)[:, None]
        j = torch.arange(k[b], device=DEV)[None, :]
        hide = j > pos
        if c["window"]:
            hide |= (pos - j >= c["window"]) & (j >= c["sinks"])
        for h in range(Hkv if n[b] else 0):
            keys, values = Kc[at, h].double(), Vc[at, h].double()
            for hq in range(h * G, h * G + G):
                x = (s["Q"][r0: r0 + n[b], hq].double() @ keys.t()) * s["scale"]
                x[hide] = -math.inf
                lse[r0: r0 + n[b], hq] = torch.logsumexp(x, 1)
                O[r0: r0 + n[b], hq] = torch.softmax(x, 1) @ values
        r0 += n[b]
    return {"O": O, "lse": lse}


def _exact_verify(s, c):
    """Request by request on the host."""
    P, Q, off = s["P"], s["Q"], s["qoff"].cpu().tolist()
    x = s["drafted"].long()
    r = torch.arange(P.shape[0], device=DEV)
    px = P[r, x].double().cpu().tolist()
    qx = Q[r, x].double().cpu().tolist() if Q is not None else [1.0] * len(px)
    x, u, v = x.cpu().tolist(), s["u"].double().cpu().tolist(), s["v"].double().cpu().tolist()
    accepted, entry, entries = [], [], [-1] * len(px)
    for b in range(c["B"]):
        a = off[b]
        while a < off[b + 1] - 1 and u[a] * qx[a] < px[a]:
            entries[a] = x[a]
            a += 1
        p = P[a].double().cpu().numpy()
        w = p
        if a < off[b + 1] - 1:
            if Q is not None:
                w = np.maximum(p - Q[a].double().cpu().numpy(), 0)
            else:
                w = p.copy()
                w[x[a]] = max(p[x[a]] - 1.0, 0.0)
            if not w.sum() > 0:
                w = p
        at = np.nonzero(w)[0]
        sums = np.cumsum(w[at])
        e = int(at[min(np.searchsorted(sums, v[b] * sums[-1], side="right"), at.size - 1)])
        entries[a] = e
        accepted.append(a - off[b])
        entry.append(e)
    i32 = lambda t: np.asarray(t, np.int32)  # noqa: E731
    return {"accepted": i32(accepted), "entry": i32(entry), "entries": i32(entries)}
