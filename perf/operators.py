"""Cross attention to an encoder's states, its gradient, and sampling of codebook entries from scores.

Each case is one call that a program makes next to the codebook lookups: it
reads the states of another sequence by attention (`attend`), trains through
that (`train`: the forward pass and the gradients), and draws an entry from
the scores of a lookup instead of taking the best one (`sample`).

`own` chooses between the operators' plain forms, written with elementary
torch operations in 32 bits (probabilities of `sample` in 64: an entry is
drawn by comparing a sum with a random number), and the library's calls.
`exact` computes the same outputs from the definitions in 64 bits.

Sizes.  Attention: B sequences of up to Lq queries and Lk encoder states, Hq
query heads over Hkv key and value heads of Dh values.  `ragged`: sequences of
different lengths, the last one of three or more with no encoder state at all;
`mask`: one state in five is masked.  Sampling: B rows of M scores.
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
        # one new token of four requests against short encoder states: latency
        {"name": "attend_token_short", "kind": "attend", "dtype": "bf16", "B": 4, "Lq": 1, "Lk": 61, "Hq": 8, "Hkv": 8,
         "Dh": 64, "ragged": False, "mask": False},
        # one new token of each request of a full serving batch, long states, heads shared by four
        {"name": "attend_token_batch", "kind": "attend", "dtype": "bf16", "B": 64, "Lq": 1, "Lk": 4000, "Hq": 32,
         "Hkv": 8, "Dh": 128, "ragged": True, "mask": False},
        # coordinates in fp32 (the library's other type), padded states under a mask
        {"name": "attend_fp32_masked", "kind": "attend", "dtype": "f32", "B": 8, "Lq": 250, "Lk": 1000, "Hq": 8,
         "Hkv": 8, "Dh": 64, "ragged": True, "mask": True},
        # whole prompts against whole documents
        {"name": "attend_prompt_large", "kind": "attend", "dtype": "bf16", "B": 4, "Lq": 4096, "Lk": 4096, "Hq": 32,
         "Hkv": 8, "Dh": 128, "ragged": False, "mask": False},
        # a training step's attention over a ragged batch with masked states and a head size between the usual ones
        {"name": "train_ragged", "kind": "train", "dtype": "bf16", "B": 5, "Lq": 333, "Lk": 777, "Hq": 12, "Hkv": 4,
         "Dh": 80, "ragged": True, "mask": True},
        # the same step at a full training batch
        {"name": "train_large", "kind": "train", "dtype": "bf16", "B": 4, "Lq": 2048, "Lk": 2048, "Hq": 16, "Hkv": 16,
         "Dh": 128, "ragged": False, "mask": False},
        # training in fp32, a small batch
        {"name": "train_fp32", "kind": "train", "dtype": "f32", "B": 2, "Lq": 200, "Lk": 500, "Hq": 8, "Hkv": 2,
         "Dh": 64, "ragged": False, "mask": False},
        # one request's next entry out of a language-sized table: latency
        {"name": "sample_one", "kind": "sample", "dtype": "f32", "B": 1, "M": 131072, "topk": True, "topp": True,
         "minp": False},
        # a serving batch over such a table, nucleus alone, scores as a bf16 product leaves them
        {"name": "sample_batch", "kind": "sample", "dtype": "bf16", "B": 200, "M": 128001, "topk": False, "topp": True,
         "minp": True},
        # temperature alone over the same batch
        {"name": "sample_temperature", "kind": "sample", "dtype": "f32", "B": 128, "M": 50257, "topk": False,
         "topp": False, "minp": False},
        # the attribute codebook of a reasoning task, every panel of every problem
        {"name": "sample_attributes", "kind": "sample", "dtype": "f32", "B": 65536, "M": 22, "topk": True, "topp": True,
         "minp": True},
        # the large compressed codebook, a batch of lookups
        {"name": "sample_codebook", "kind": "sample", "dtype": "f32", "B": 8192, "M": 2048, "topk": True, "topp": True,
         "minp": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "train", "sample", "sample"])
    if kind == "sample":
        M = _log(rng, 2, 131072)
        B = _log(rng, 1, max(1, min(65536, (1 << 24) // M)))
        return {"kind": kind, "dtype": rng.choice(["f32", "bf16"]), "B": B, "M": M, "topk": rng.random() < 0.5,
                "topp": rng.random() < 0.6, "minp": rng.random() < 0.3}
    dtype = rng.choice(["bf16", "bf16", "f32"])
    Dh = rng.choice([32, 40, 64, 64, 72, 96, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    Hq = Hkv * rng.choice([1, 1, 2, 3, 4])
    most = 1 << (30 if kind == "attend" else 27)        # B Hq Lq Lk
    if dtype == "f32":
        most >>= 3
    if kind == "attend" and rng.random() < 0.4:
        Lq = rng.choice([1, 1, 1, 2, 5])
        Lk = _log(rng, 1, 16384)
    else:
        Lq = _log(rng, 2, 2048)
        Lk = _log(rng, 8, 4096)
    B = _log(rng, 1, max(1, min(64, most // (Hq * Lq * Lk), (1 << 28) // (Hkv * Lk * Dh))))
    return {"kind": kind, "dtype": dtype, "B": B, "Lq": Lq, "Lk": Lk, "Hq": Hq, "Hkv": Hkv, "Dh": Dh,
            "ragged": rng.random() < 0.5, "mask": rng.random() < 0.4}


def lengths(c):
    """Lengths of the sequences (a case's own, whatever the seed)."""
    B, Lq, Lk = c["B"], c["Lq"], c["Lk"]
    if not c["ragged"]:
        return [Lq] * B, [Lk] * B
    ql = [Lq - (13 * b) % Lq for b in range(B)]
    kl = [Lk - (97 * b) % Lk for b in range(B)]
    if B > 2:
        kl[B - 1] = 0
    return ql, kl


def work(c):
    if c["kind"] == "sample":
        e = 2 if c["dtype"] == "bf16" else 4
        # scores, random number and the three parameters read; index, probability and count written;
        # per score a comparison, a scaled difference, an exponential (one operation) and a sum
        return {"bytes": c["B"] * (c["M"] * e + 16 + 12), "flops": 4 * c["B"] * c["M"]}
    e = 2 if c["dtype"] == "bf16" else 4
    ql, kl = lengths(c)
    seen = 0.8 if c["mask"] else 1.0
    q = sum(ql) * c["Hq"] * c["Dh"]
    kv = int(seen * sum(kl)) * c["Hkv"] * c["Dh"]
    pairs = seen * sum(a * b for a, b in zip(ql, kl)) * c["Hq"] * c["Dh"]
    lens = 8 * c["B"] + (c["B"] * c["Lk"] if c["mask"] else 0)
    rows = c["B"] * c["Lq"] * c["Hq"]
    if c["kind"] == "attend":       # Q, K, V read, O and the row statistics written; two products
        return {"bytes": e * (q + 2 * kv + rows * c["Dh"]) + 4 * rows + lens, "flops": int(4 * pairs)}
    # the forward pass; then Q, K, V, O, dO and the statistics read, three gradients written; five products
    every = c["B"] * c["Lk"] * c["Hkv"] * c["Dh"]
    back = e * (q * 3 + 2 * kv + rows * c["Dh"] + 2 * every) + 4 * rows
    return {"bytes": e * (q + 2 * kv + rows * c["Dh"]) + 4 * rows + back + lens, "flops": int(14 * pairs)}


# ------------------------------------------------------------------ inputs

def prepare(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"case": dict(c)}
    if c["kind"] == "sample":
        B, M = c["B"], c["M"]
        S = torch.randn(B, M, generator=g, device=DEV) * 2.5
        # entries that a grammar forbids
        S.masked_fill_(torch.rand(B, M, generator=g, device=DEV) < 0.05, -math.inf)
        s["S"] = S.to(DT[c["dtype"]])
        s["u"] = torch.rand(B, generator=g, device=DEV)
        pick = lambda lo, hi: lo + (hi - lo) * torch.rand(B, generator=g, device=DEV)  # noqa: E731
        s["temperature"] = pick(0.5, 1.2)
        s["top_k"] = torch.randint(1, 101, (B,), generator=g, device=DEV, dtype=torch.int32) if c["topk"] else None
        s["top_p"] = pick(0.7, 0.98) if c["topp"] else None
        s["min_p"] = pick(0.0, 0.1) if c["minp"] else None
        return s
    dt = DT[c["dtype"]]
    B, Lq, Lk, Hq, Hkv, Dh = (c[k] for k in ("B", "Lq", "Lk", "Hq", "Hkv", "Dh"))
    normal = lambda *n: torch.randn(*n, generator=g, device=DEV).to(dt)  # noqa: E731
    s["Q"], s["K"], s["V"] = normal(B, Lq, Hq, Dh), normal(B, Lk, Hkv, Dh), normal(B, Lk, Hkv, Dh)
    if c["kind"] == "train":
        s["dO"] = normal(B, Lq, Hq, Dh)
    ql, kl = lengths(c)
    s["qlen"] = torch.tensor(ql, dtype=torch.int32, device=DEV) if c["ragged"] else None
    s["klen"] = torch.tensor(kl, dtype=torch.int32, device=DEV) if c["ragged"] else None
    s["mask"] = torch.rand(B, Lk, generator=g, device=DEV) < 0.8 if c["mask"] else None
    s["scale"] = 1.0 / math.sqrt(Dh)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    if kind == "sample":
        return _plain_sample(s)
    return _plain_attend(s, kind == "train")


def _run_own(s):
    from paper_2608_01528_amd import gramspace as gs

    c = s["case"]
    if c["kind"] == "sample":
        p = {k: s[k] for k in ("temperature", "top_k", "top_p", "min_p") if s[k] is not None}
        idx, prob, kept = gs.gs_sample(s["S"], s["u"], prob=True, kept=True, **p)
        return {"idx": idx, "prob": prob, "kept": kept}
    given = {"qlen": s["qlen"], "klen": s["klen"], "mask": s["mask"], "scale": s["scale"]}
    O, lse = gs.gs_cross_attention(s["Q"], s["K"], s["V"], lse=True, **given)
    if c["kind"] == "attend":
        return {"O": O, "lse": lse}
    dQ, dK, dV = gs.gs_cross_attention_grad(s["dO"], s["Q"], s["K"], s["V"], O, lse, **given)
    return {"O": O, "lse": lse, "dQ": dQ, "dK": dK, "dV": dV}


def _plain_attend(s, train):
    """O = softmax(scale Q K^T) V over the states that a sequence has, in fp32; with `train` the gradients of
    sum(O dO) too: dV = P^T dO, dS = P (dO V^T - rowsum(dO O)), dQ = scale dS K, dK = scale dS^T Q."""
    c = s["case"]
    B, Lq, Lk, Hq, Hkv, Dh = (c[k] for k in ("B", "Lq", "Lk", "Hq", "Hkv", "Dh"))
    G = Hq // Hkv
    dt, dev = s["Q"].dtype, s["Q"].device

    def rows(t):        # (B, Lq, Hq, Dh) -> (B Hkv, G Lq, Dh)
        return t.float().reshape(B, Lq, Hkv, G, Dh).permute(0, 2, 3, 1, 4).reshape(B * Hkv, G * Lq, Dh)

    def back(t):
        return t.reshape(B, Hkv, G, Lq, Dh).permute(0, 3, 1, 2, 4).reshape(B, Lq, Hq, Dh).to(dt)

    def states(t, live):    # (B, Lk, Hkv, Dh) -> (B Hkv, Lk, Dh), masked states as zeros
        if live is not None:
            t = torch.where(live[:, :, None, None], t, torch.zeros((), dtype=dt, device=dev))
        return t.float().permute(0, 2, 1, 3).reshape(B * Hkv, Lk, Dh)

    def unstates(t):
        return t.reshape(B, Hkv, Lk, Dh).permute(0, 2, 1, 3).contiguous().to(dt)

    live = None
    if s["klen"] is not None:
        live = torch.arange(Lk, device=dev)[None, :] < s["klen"][:, None]
    if s["mask"] is not None:
        live = s["mask"] if live is None else live & s["mask"]
    q, k, v = rows(s["Q"]), states(s["K"], live), states(s["V"], live)
    P = torch.matmul(q, k.transpose(1, 2)).mul_(s["scale"]).view(B, Hkv, G, Lq, Lk)
    if live is not None:
        P.masked_fill_(~live[:, None, None, None, :], -math.inf)
    if s["qlen"] is not None:
        there = torch.arange(Lq, device=dev)[None, :] < s["qlen"][:, None]
        P.masked_fill_(~there[:, None, None, :, None], -math.inf)
    m = P.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P.sub_(m).exp_()
    l = P.sum(dim=-1, keepdim=True)
    lse = (m + l.log()).squeeze(-1).permute(0, 1, 2, 3).reshape(B, Hq, Lq)
    P.div_(torch.where(l == 0, torch.ones_like(l), l))
    P = P.view(B * Hkv, G * Lq, Lk)
    o = torch.matmul(P, v)
    out = {"O": back(o), "lse": lse}
    if train:
        do = rows(s["dO"])
        if s["qlen"] is not None:
            do = do * there[:, None, None, :].expand(B, Hkv, G, Lq).reshape(B * Hkv, G * Lq, 1)
        dS = torch.matmul(do, v.transpose(1, 2))
        dS.sub_((do * o).sum(dim=-1, keepdim=True)).mul_(P)
        out["dQ"] = back(torch.matmul(dS, k).mul_(s["scale"]))
        out["dK"] = unstates(torch.matmul(dS.transpose(1, 2), q).mul_(s["scale"]))
        out["dV"] = unstates(torch.matmul(P.transpose(1, 2), do))
    return out


def _plain_sample(s):
    """Entries in falling order of their scores (equal scores by index); weights exp((x - max) / temperature); the
    first top_k of them; of these as many as are needed for top_p of their weight; of these the ones with at least
    min_p of the largest weight.  The entry drawn is the first, by index, at which the sum of the kept weights
    passes u times their total."""
    S, u = s["S"], s["u"].double()
    B, M = S.shape
    x, order = torch.sort(S, dim=1, descending=True, stable=True)
    w = torch.exp((x.double() - x[:, :1].double()) / s["temperature"].double()[:, None])
    place = torch.arange(M, device=S.device)[None, :]
    keep = x > -math.inf
    if s["top_k"] is not None:
        keep &= place < s["top_k"][:, None]
    if s["top_p"] is not None:
        wk = w * keep
        before = wk.cumsum(1) - wk
        keep &= (before < s["top_p"].double()[:, None] * wk.sum(1, keepdim=True)) | (place == 0)
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    w = torch.zeros_like(w).scatter_(1, order, w * keep)
    c = w.cumsum(1)
    hit = (c > u[:, None] * c[:, -1:]) & (w > 0)
    idx = torch.where(hit, place, M).amin(1)
    kept = keep.sum(1)
    prob = w.gather(1, idx[:, None].clamp(max=M - 1))[:, 0] / c[:, -1]
    none = kept == 0
    return {"idx": torch.where(none, -1, idx).int(), "prob": torch.where(none, 0.0, prob).float(), "kept": kept.int()}


# ------------------------------------------------------------------ 64 bits, from the definitions

def exact(c, seed):
    s = prepare(c, seed)
    return _exact_sample(s) if c["kind"] == "sample" else _exact_attend(s, c)


def _exact_attend(s, c):
    """Sequence by sequence and head by head over the states that are there; gradients by differentiation."""
    B, Lq, Lk, Hq, Hkv, Dh = (c[k] for k in ("B", "Lq", "Lk", "Hq", "Hkv", "Dh"))
    if B * Hq > 4096:
        return None
    train = c["kind"] == "train"
    ql, kl = lengths(c)
    f64 = dict(dtype=torch.float64, device=DEV)
    O, lse = torch.zeros(B, Lq, Hq, Dh, **f64), torch.full((B, Hq, Lq), -math.inf, **f64)
    grads = [torch.zeros(s[n].shape, **f64) for n in "QKV"] if train else None
    for b in range(B):
        at = torch.arange(kl[b], device=DEV)
        if s["mask"] is not None:
            at = at[s["mask"][b, : kl[b]]]
        if at.numel() == 0:
            continue
        for h in range(Hq):
            j = h // (Hq // Hkv)
            q = s["Q"][b, : ql[b], h].double().requires_grad_(train)
            k = s["K"][b, at, j].double().requires_grad_(train)
            v = s["V"][b, at, j].double().requires_grad_(train)
            logits = s["scale"] * (q @ k.t())
            o = torch.softmax(logits, dim=1) @ v
            O[b, : ql[b], h] = o.detach()
            lse[b, h, : ql[b]] = torch.logsumexp(logits, dim=1).detach()
            if train:
                d = torch.autograd.grad(o, (q, k, v), s["dO"][b, : ql[b], h].double())
                grads[0][b, : ql[b], h] = d[0]
                grads[1][b, at, j] += d[1]
                grads[2][b, at, j] += d[2]
    out = {"O": O, "lse": lse}
    if train:
        out.update(dQ=grads[0], dK=grads[1], dV=grads[2])
    return out


def _exact_sample(s):
    """Row by row on the host: a row's entries ranked, cut three times, and searched by their running sum."""
    host = {k: None if s[k] is None else s[k].double().cpu().numpy() for k in
            ("S", "u", "temperature", "top_k", "top_p", "min_p")}
    S = host["S"]
    B, M = S.shape
    idx, prob, kept = np.full(B, -1, np.int32), np.zeros(B, np.float64), np.zeros(B, np.int32)
    for b in range(B):
        row = S[b]
        order = np.argsort(-row, kind="stable")
        order = order[: np.count_nonzero(row > -np.inf)]
        if not order.size:
            continue
        if host["top_k"] is not None:
            order = order[: int(host["top_k"][b])]
        w = np.exp((row[order] - row[order[0]]) / host["temperature"][b])
        if host["top_p"] is not None:
            reached = np.nonzero(np.cumsum(w) >= host["top_p"][b] * w.sum())[0]
            n = reached[0] + 1 if reached.size else order.size
            order, w = order[:n], w[:n]
        if host["min_p"] is not None:
            n = max(1, np.count_nonzero(w >= host["min_p"][b]))
            order, w = order[:n], w[:n]
        by = np.argsort(order)
        order, w = order[by], w[by]
        sums = np.cumsum(w)
        i = min(np.searchsorted(sums, host["u"][b] * sums[-1], side="right"), order.size - 1)
        idx[b], prob[b], kept[b] = order[i], w[i] / sums[-1], order.size
    return {"idx": idx, "prob": prob, "kept": kept}
