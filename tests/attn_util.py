"""Cross attention in 64 bits, with a bound of what the kernels' arithmetic may
be off by, element by element.

u = 2^-24 is half an fp32 step, v half a step of the tensors' type (bf16 2^-8,
fp32 2^-24).  Per score the fp32 dot product, its scaling and the exponent are
off by at most

  dS = (Dh + 4) u scale sum_d |q_d k_d| + 4 u |S|

and a probability by the factor 1 + e, e = 2 max_j dS + 8 u + 3 u |lse| (its
exponent and that of the sum, or the stored lse).  Sums over n terms are off by
n u of the terms' absolute sum at most, whatever their order; rescaling a
running sum adds two roundings a tile.  A value that enters a product in the
tensors' type is off by v more, and so is an output.  Numbers below the normal
ones (F = 2^-126) may count as zero wherever they arise: a probability (F off,
F more as it enters a product), its gradient, and each term of a product; a
sum of n products p w of such p is off by 2 F sum |w| + n F then.
"""
import torch

U = 2.0 ** -24
F = 2.0 ** -126
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def reference(Q, K, V, qlen=None, klen=None, mask=None, scale=None, dO=None):
    """Returns {name: (value, bound)} in float64 on the CPU; tensors of the
    given shapes (any device and strides)."""
    v = HALF[Q.dtype]
    cpu = lambda t: None if t is None else t.detach().cpu()  # noqa: E731
    Q, K, V, dO, qlen, klen, mask = (cpu(t) for t in (Q, K, V, dO, qlen, klen, mask))
    B, Lq, Hq, Dh = Q.shape
    Lk, Hkv = K.shape[1:3]
    G = Hq // Hkv
    scale = Dh ** -0.5 if scale is None else scale
    z = lambda *n: torch.zeros(*n, dtype=torch.float64)  # noqa: E731
    out = {"O": [z(B, Lq, Hq, Dh), z(B, Lq, Hq, Dh)],
           "lse": [torch.full((B, Hq, Lq), -float("inf"), dtype=torch.float64), z(B, Hq, Lq)]}
    if dO is not None:
        for n, t in (("dQ", Q), ("dK", K), ("dV", V)):
            out[n] = [z(*t.shape), z(*t.shape)]
    for b in range(B):
        nq = Lq if qlen is None else min(max(int(qlen[b]), 0), Lq)
        nk = Lk if klen is None else min(max(int(klen[b]), 0), Lk)
        at = torch.arange(nk)
        if mask is not None:
            at = at[mask[b, :nk] != 0]
        if not at.numel() or not nq:
            continue
        n = at.numel()
        for h in range(Hq):
            j = h // G
            q, k, w = Q[b, :nq, h].double(), K[b, at, j].double(), V[b, at, j].double()
            S = scale * (q @ k.t())
            dS = (Dh + 4) * U * abs(scale) * (q.abs() @ k.abs().t()) + 4 * U * S.abs()
            lse = torch.logsumexp(S, 1)
            P = torch.exp(S - lse[:, None])
            slip = dS.amax(1)
            e = (2 * slip + 8 * U + 3 * U * lse.abs())[:, None]
            e = torch.expm1(e)
            sums = (2 * n + 64) * U
            o, A = P @ w, P @ w.abs()
            tol_o = A * (v * (1 + e) + e + 2 * sums) + 2 * F * w.abs().sum(0) + n * F
            o_out = tol_o + v * (o.abs() + tol_o)
            out["O"][0][b, :nq, h], out["O"][1][b, :nq, h] = o, o_out
            out["lse"][0][b, h, :nq] = lse
            out["lse"][1][b, h, :nq] = slip + sums + 8 * U * (1 + lse.abs())
            if dO is None:
                continue
            d = dO[b, :nq, h].double()
            dP, adP = d @ w.t(), d.abs() @ w.abs().t()
            D = (d * o).sum(1, keepdim=True)
            tol_D = (d.abs() * o_out).sum(1, keepdim=True) + (Dh + 2) * U * (d.abs() * (o.abs() + o_out)).sum(1, keepdim=True)
            g = P * (dP - D)
            tol_dP = (Dh + 2) * U * adP + 2 * U * (dP.abs() + D.abs())
            tol_g = P * (1 + e) * (tol_dP + tol_D) + g.abs() * e + F * (adP + D.abs() + tol_dP + tol_D)
            tol_g = tol_g + (v + 2 * U) * (g.abs() + tol_g) + 2 * F
            for name, rows, val, err in (
                    ("dQ", (b, slice(0, nq), h), scale * (g @ k), abs(scale) * (tol_g @ k.abs() + 2 * n * U * (g.abs() @ k.abs())) + n * F),
                    ("dK", (b, at, j), scale * (g.t() @ q), abs(scale) * (tol_g.t() @ q.abs() + 2 * G * nq * U * (g.abs().t() @ q.abs())) + nq * F),
                    ("dV", (b, at, j), P.t() @ d, (P * (e + (v + 2 * U) * (1 + e))).t() @ d.abs() + 2 * G * nq * U * (P.t() @ d.abs())
                     + 2 * F * d.abs().sum(0) + nq * F)):
                out[name][0][rows] += val
                out[name][1][rows] += err
    # the outputs' own rounding (an fp32 result takes a few more steps on its way out)
    for name in ("dQ", "dK", "dV"):
        if name in out:
            out[name][1] += (v + 2 * U) * (out[name][0].abs() + out[name][1])
    return {n: (a, t + F) for n, (a, t) in out.items()}


def check(got, ref, name):
    """Every element within its bound (infinities equal)."""
    value, bound = ref[name]
    g = got.detach().cpu().double()
    assert g.shape == value.shape, (name, g.shape, value.shape)
    fine = torch.isfinite(value)
    assert torch.equal(g[~fine], value[~fine]), name
    off = (g[fine] - value[fine]).abs()
    over = ~(off <= bound[fine])
    assert not over.any(), "%s: %d of %d beyond the bound, worst %.3g against %.3g" % (
        name, int(over.sum()), over.numel(), float(off[over].max()), float(bound[fine][over].max()))
