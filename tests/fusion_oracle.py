"""Attention-based fusion in 64 bits, from the formulas: rotary positions, norms per head, attention of ragged sequences.

Everything takes and returns float64 torch tensors on the CPU (numpy-like loops over sequences; no code of the library).  The
*_bound functions give, element by element, how far a result formed in 32 bits and rounded once to its type may be off.
"""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}     # a rounding is off by at most half a step, relative


def frequencies(rot, base=10000.0, factor=1.0, trained=0.0, low=1.0, high=32.0):
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    keep = ((trained * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1) if factor != 1.0 else torch.ones_like(f)
    return f * (keep + (1 - keep) / factor)


def rotate(x, heads, freqs, pos, scale=1.0, interleaved=False, inverse=False):
    x = x.reshape(x.shape[0], heads, -1)
    y, half = x.clone(), freqs.numel()
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    t = pos.double()[:, None, None] * freqs
    t = -t if inverse else t
    y[..., a] = scale * (x[..., a] * t.cos() - x[..., b] * t.sin())
    y[..., b] = scale * (x[..., b] * t.cos() + x[..., a] * t.sin())
    return y.flatten(1)


def rotate_scale(x, heads, freqs, scale, interleaved):
    """|x_a| + |x_b| of every element's pair (times scale), |x| of what is not rotated: the size of the terms of a result."""
    x = x.abs().reshape(x.shape[0], heads, -1)
    y, half = x.clone(), freqs.numel()
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    y[..., a] = y[..., b] = scale * (x[..., a] + x[..., b])
    return y.flatten(1)


def norm(x, heads, w, eps):
    x = x.reshape(x.shape[0], heads, -1)
    return (x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w).flatten(1)


def norm_rotary_backward(dy, x, heads, w, eps, freqs, pos, scale=1.0, interleaved=False):
    """dx, dw, and the sizes of the terms behind them."""
    u = rotate(dy, heads, freqs, pos, scale, interleaved, inverse=True).reshape(x.shape[0], heads, -1)
    us = rotate_scale(dy, heads, freqs, scale, interleaved).reshape(x.shape[0], heads, -1)
    x = x.reshape(x.shape[0], heads, -1)
    rms = (x.square().mean(-1, keepdim=True) + eps).sqrt()
    n = x / rms
    dx = (u * w - n * (u * w * n).mean(-1, keepdim=True)) / rms
    dx_terms = (us * w.abs() + n.abs() * (us * (w * n).abs()).mean(-1, keepdim=True)) / rms
    return dx.flatten(1), (u * n).sum((0, 1)), dx_terms.flatten(1), (us * n.abs()).sum((0, 1))


def attention(q, k, v, q_ptr, k_ptr, heads, kv_heads, scale, mask=None, dout=None, dtype=torch.float32, rounded_p=False, weights=False):
    """Forward (and with dout backward) pass, and bounds.  Returns dict name -> (value, bound) for out, lse, dq, dk, dv.

    Bounds, with h half a step of the type and e = 2^-24: a score is a sum of head_dim products in 32 bits and is off by
    ds <= (head_dim + 2) e scale |q| . |k|; p = exp(score - lse) therefore by a factor 1 + dp, dp <= 2 max ds + 2^-20 (score, lse, the
    hardware's exponential, its argument's rounding up to 2^7 in size: 2^7 e = 2^-17 is added where scores are that large); with
    rounded_p also by h, as p goes into the products in 16 bits.  A sum of n such terms adds n e of their absolute sum.  The backward
    pass reads `out` as it was stored (off by its own bound).  A p below 2^-126 has no normal 32-bit value: it may count as zero, so p is
    off by tiny = 2^-126 on top, and every result by tiny times the sum of what p multiplies."""
    G, hd = heads // kv_heads, q.shape[1] // heads
    e, h = 2.0 ** -24, HALF[dtype]
    hp, tiny = HALF[torch.bfloat16] if rounded_p else 0.0, 2.0 ** -126
    z = torch.zeros
    out, out_b = z(q.shape, dtype=torch.float64), z(q.shape, dtype=torch.float64)
    lse, lse_b = torch.full((q.shape[0], heads), -math.inf, dtype=torch.float64), z(q.shape[0], heads, dtype=torch.float64)
    grads = {n: (torch.zeros_like(t), torch.zeros_like(t)) for n, t in (("dq", q), ("dk", k), ("dv", v))}
    for s in range(len(q_ptr) - 1):
        rq = slice(int(q_ptr[s]), int(q_ptr[s + 1]))
        seen = torch.arange(int(k_ptr[s]), int(k_ptr[s + 1]))
        if mask is not None:
            seen = seen[mask[seen] != 0]
        if rq.start == rq.stop or not seen.numel():
            continue
        n = seen.numel()
        qs, ks, vs = q[rq].view(-1, kv_heads, G, hd), k[seen].view(-1, kv_heads, hd), v[seen].view(-1, kv_heads, hd)
        sc = torch.einsum("qhgd,khd->hgqk", qs, ks) * scale
        ds_ = (hd + 2) * e * scale * torch.einsum("qhgd,khd->hgqk", qs.abs(), ks.abs())
        l = torch.logsumexp(sc, -1, keepdim=True)
        p = torch.exp(sc - l)
        worst = ds_.amax(-1, keepdim=True) + e * sc.abs().amax(-1, keepdim=True)
        dp_ = 2 * worst + 2.0 ** -20 + n * e
        o = torch.einsum("hgqk,khd->qhgd", p, vs)
        ob = h * o.abs() + torch.einsum("hgqk,khd->qhgd", p * (dp_ + hp + n * e) + tiny, vs.abs()) * (1 + h) + tiny
        out[rq], out_b[rq] = o.flatten(1), ob.flatten(1)
        lse[rq] = l[..., 0].permute(2, 0, 1).flatten(1)
        lse_b[rq] = (worst[..., 0] + 2.0 ** -20 + n * e + 2 * e * l[..., 0].abs()).permute(2, 0, 1).flatten(1)
        if dout is None:
            continue
        g = dout[rq].view(-1, kv_heads, G, hd)
        dpv = torch.einsum("qhgd,khd->hgqk", g, vs)
        D = torch.einsum("qhgd,qhgd->hgq", g, o)[..., None]
        # what p, dP and D may be off by, and with them dS = p (dP - D)
        dD = torch.einsum("qhgd,qhgd->hgq", g.abs(), ob + (hd + 2) * e * o.abs())[..., None]
        ddp = (hd + 2) * e * torch.einsum("qhgd,khd->hgqk", g.abs(), vs.abs())
        dS = p * (dpv - D)
        dSb = dS.abs() * (dp_ + hp) + p * (ddp + dD) * (1 + dp_ + hp) + tiny * (1 + (dpv - D).abs())
        nq = qs.shape[0] * G
        for name, val, bound, terms, rows in (
                ("dv", torch.einsum("hgqk,qhgd->khd", p, g), torch.einsum("hgqk,qhgd->khd", p * (dp_ + hp) + tiny, g.abs()),
                 torch.einsum("hgqk,qhgd->khd", p, g.abs()) * nq * e, seen),
                ("dq", torch.einsum("hgqk,khd->qhgd", dS, ks) * scale, torch.einsum("hgqk,khd->qhgd", dSb, ks.abs()) * scale,
                 torch.einsum("hgqk,khd->qhgd", dS.abs(), ks.abs()) * scale * (n + 2) * e, rq),
                ("dk", torch.einsum("hgqk,qhgd->khd", dS, qs) * scale, torch.einsum("hgqk,qhgd->khd", dSb, qs.abs()) * scale,
                 torch.einsum("hgqk,qhgd->khd", dS.abs(), qs.abs()) * scale * (nq + 2) * e, seen)):
            grads[name][0][rows] = val.flatten(1)
            grads[name][1][rows] = (h * val.abs() + (bound + terms) * (1 + h) + tiny).flatten(1)
    res = {"out": (out, out_b), "lse": (lse, lse_b)}
    if dout is not None:
        res.update(grads)
    return res
