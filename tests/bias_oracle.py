"""Attention of ragged sequences with a bias by head and bucket of the distance, in 64 bits from the formulas, on the CPU (no code of the
library).  Values come with bounds: how far, element by element, a result formed in 32 bits and rounded once to its type may be off."""
import math

import torch

E = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}     # a rounding is off by at most half a step, relative
HIDES = -1.0e30


def edges(buckets, far, both=False):
    """Ascending edges: bucket numbers up to buckets / 2 are distances, from there on evenly by the logarithm up to far."""
    half, side = max(buckets // 2, 1), []
    for i in range(1, buckets):
        t = i
        if i >= half:
            x = half * (max(far, half + 1) / half) ** ((i - half) / max(buckets - half, 1))
            t = round(x) if abs(x - round(x)) < 1e-9 * x else math.ceil(x)
        side.append(max(t, side[-1] + 1 if side else 1))
    return [1 - t for t in reversed(side)] + (side if both else [])


def buckets(edge, pos_q, pos_k):
    """[queries, keys]: how many edges are not above pos_k - pos_q."""
    apart = pos_k.long()[None, :] - pos_q.long()[:, None]
    return (apart[..., None] >= edge.long()).sum(-1)


def attention(q, k, v, q_ptr, k_ptr, heads, kv_heads, scale, edge, table, pos_q=None, pos_k=None, mask=None, dout=None, dtype=torch.float32,
              rounded_p=False):
    """Forward (and with dout backward) pass.  Returns dict name -> (value, bound) for out, lse, dq, dk, dv, dtable.

    Bounds, with h half a step of the type and e = 2^-24: a score is a sum of head_dim products in 32 bits and a bias, off by
    (head_dim + 2) e scale |q| . |k| + 4 e (|scale q . k| + |bias|); p = exp(score - lse) is off by a factor 1 + dp, dp <= 2 max of that +
    e max |score| + 2^-20 (the hardware's exponential) + n e; with rounded_p also by half a step of bf16, as p goes into products.  Sums of n
    terms add n e of their absolute sum.  The backward pass reads `out` as it was stored, which dtable does not see: D = sum p dP there, with
    p and dP in 32 bits.  A p below 2^-126 may count as zero."""
    G, hd = heads // kv_heads, q.shape[1] // heads
    h, tiny = HALF[dtype], 2.0 ** -126
    hp = HALF[torch.bfloat16] if rounded_p else 0.0
    bias = torch.where(table.double() <= HIDES, -math.inf, table.double())
    res = {n: (torch.zeros_like(t), torch.zeros_like(t)) for n, t in (("out", q), ("dq", q), ("dk", k), ("dv", v))}
    res["dtable"] = torch.zeros_like(bias), torch.zeros_like(bias)
    res["lse"] = torch.full((q.shape[0], heads), -math.inf, dtype=torch.float64), torch.zeros(q.shape[0], heads, dtype=torch.float64)
    chain = 0
    table_terms = torch.zeros_like(bias)
    for s in range(len(q_ptr) - 1):
        rq, k0 = slice(int(q_ptr[s]), int(q_ptr[s + 1])), int(k_ptr[s])
        seen = torch.arange(k0, int(k_ptr[s + 1]))
        if mask is not None:
            seen = seen[mask[seen] != 0]
        if rq.start == rq.stop or not seen.numel():
            continue
        n, rows = seen.numel(), rq.stop - rq.start
        at_q = torch.arange(rows) if pos_q is None else pos_q[rq]
        at_k = seen - k0 if pos_k is None else pos_k[seen]
        where = buckets(edge, at_q, at_k)
        b = bias[where].permute(2, 0, 1).reshape(kv_heads, G, rows, n)
        qs, ks, vs = q[rq].view(-1, kv_heads, G, hd), k[seen].view(-1, kv_heads, hd), v[seen].view(-1, kv_heads, hd)
        dots = torch.einsum("qhgd,khd->hgqk", qs, ks) * scale
        on = torch.isfinite(b)
        sc = dots + b
        size = torch.where(on, dots.abs() + b.abs(), torch.zeros_like(b))
        off = (hd + 2) * E * scale * torch.einsum("qhgd,khd->hgqk", qs.abs(), ks.abs()) + 4 * E * size
        l = torch.logsumexp(sc, -1, keepdim=True)
        dead = l == -math.inf
        p = torch.where(dead, torch.zeros_like(sc), torch.exp(sc - torch.where(dead, torch.zeros_like(l), l)))
        worst = off.amax(-1, keepdim=True) + E * size.amax(-1, keepdim=True)
        dp = 2 * worst + 2.0 ** -20 + n * E
        o = torch.einsum("hgqk,khd->qhgd", p, vs)
        ob = h * o.abs() + torch.einsum("hgqk,khd->qhgd", p * (dp + hp + n * E) + tiny, vs.abs()) * (1 + h) + tiny
        res["out"][0][rq], res["out"][1][rq] = o.flatten(1), ob.flatten(1)
        lse_b = torch.where(dead, torch.zeros_like(l), worst + 2.0 ** -20 + n * E + 2 * E * l.abs())[..., 0]
        res["lse"][0][rq], res["lse"][1][rq] = l[..., 0].permute(2, 0, 1).flatten(1), lse_b.permute(2, 0, 1).flatten(1)
        if dout is None:
            continue
        g = dout[rq].view(-1, kv_heads, G, hd)
        dpv = torch.einsum("qhgd,khd->hgqk", g, vs)
        D = (p * dpv).sum(-1, keepdim=True)
        dD = torch.einsum("qhgd,qhgd->hgq", g.abs(), ob + (hd + 2) * E * o.abs())[..., None]
        ddp = (hd + 2) * E * torch.einsum("qhgd,khd->hgqk", g.abs(), vs.abs())
        dS = p * (dpv - D)
        dSb = dS.abs() * (dp + hp) + p * (ddp + dD) * (1 + dp + hp) + tiny * (1 + (dpv - D).abs())
        nq = rows * G
        for name, val, bound, terms, to in (
                ("dv", torch.einsum("hgqk,qhgd->khd", p, g), torch.einsum("hgqk,qhgd->khd", p * (dp + hp) + tiny, g.abs()),
                 torch.einsum("hgqk,qhgd->khd", p, g.abs()) * nq * E, seen),
                ("dq", torch.einsum("hgqk,khd->qhgd", dS, ks) * scale, torch.einsum("hgqk,khd->qhgd", dSb, ks.abs()) * scale,
                 torch.einsum("hgqk,khd->qhgd", dS.abs(), ks.abs()) * scale * (n + 2) * E, rq),
                ("dk", torch.einsum("hgqk,qhgd->khd", dS, qs) * scale, torch.einsum("hgqk,qhgd->khd", dSb, qs.abs()) * scale,
                 torch.einsum("hgqk,qhgd->khd", dS.abs(), qs.abs()) * scale * (nq + 2) * E, seen)):
            res[name][0][to] = val.flatten(1)
            res[name][1][to] = (h * val.abs() + (bound + terms) * (1 + h) + tiny).flatten(1)
        # D formed anew: a mean of dP by p, each off by ddp and p's factor, which the mean has in common
        dDt = (p * (ddp + (dpv - D).abs() * dp)).sum(-1, keepdim=True) + (n + 4) * E * (p * dpv.abs()).sum(-1, keepdim=True)
        part = dS.abs() * dp + p * (ddp + dDt) * (1 + dp) + tiny * (1 + (dpv - D).abs())
        flat = where.reshape(-1)
        pairs = lambda t: t.reshape(heads, -1).T
        res["dtable"][0].index_add_(0, flat, pairs(dS))
        res["dtable"][1].index_add_(0, flat, pairs(part))
        table_terms.index_add_(0, flat, pairs(dS.abs()))
        chain = max(chain, n) + rows
    res["dtable"][1].add_((chain + 64) * E * table_terms)
    return res
