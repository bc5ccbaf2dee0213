"""Dropout and layer norm in 64 bits, from the formulas, on the CPU (no code of the library).

The *_bound values give, element by element, how far a result formed in 32 bits and rounded once to its type may be off."""
import numpy as np
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}     # a rounding is off by at most half a step, relative
E = 2.0 ** -24


def philox(c, k):
    """Philox4x32-10 of counters c (4 arrays of uint64 below 2^32) and a key (2 numbers)."""
    c, k = [np.asarray(x, dtype=np.uint64) for x in c], list(k)
    low, s = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> s) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> s) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def cut(p):
    return min(int(p * 65536 + 0.5), 65535)


def factors(rows, dim, p, seed, place=0, step=0):
    """What every element of a [rows, dim] matrix is multiplied by: 0 or 2^16 / (2^16 - t), float64."""
    unit, row = np.meshgrid(np.arange((dim + 7) // 8), np.arange(rows))
    w = philox((unit, row, np.full_like(unit, 0x80000000 | place), np.full_like(unit, step & 0xFFFFFFFF)), (seed & 0xFFFFFFFF, seed >> 32))
    halves = np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], -1).reshape(rows, (dim + 7) // 8 * 8)[:, :dim]
    t = cut(p)
    return torch.from_numpy(np.where(halves < t, 0.0, 65536.0 / (65536 - t)))


def total(x, r, f):
    """residual + dropout(x), and how far the same in 32 bits may be off.  A dropped element is 0 whatever it holds."""
    d = torch.where(f == 0, torch.zeros_like(x), x * f)
    z = d if r is None else d + r
    return z, 3 * E * (d.abs() + (0 if r is None else r.abs()))


def norm(x, r, f, gain, shift, eps, dtype, dy=None, dz_in=None):
    """Layer norm of residual + dropout(x).  Returns dict name -> (value, bound).

    A sum over a row is a chain of at most 32 additions in a thread and 8 more across threads, with the products and the division by the
    width about 48 roundings: 48 E of its absolute terms.  The variance is a mean of squares of z - m; 1 / sqrt is off by 2^-22 at most."""
    z, bz = total(x, r, f)
    m = z.mean(-1, keepdim=True)
    bm = 48 * E * z.abs().mean(-1, keepdim=True) + bz.mean(-1, keepdim=True)
    d = z - m
    bd = bz + bm + E * d.abs()
    var = d.square().mean(-1, keepdim=True)
    s = (var + eps) ** -0.5
    rel = 48 * E + 2.0 ** -22 + (d.abs() * bd + bd.square()).mean(-1, keepdim=True) * s * s       # of s: half of what the variance has
    n = d * s
    bn = bd * s + n.abs() * (rel + 2 * E)
    h, one = HALF[dtype], torch.ones_like(z)
    g = one if gain is None else one * gain
    y = n * g + (0 if shift is None else shift)
    res = {"y": (y, h * y.abs() + (1 + h) * (g.abs() * bn + 2 * E * ((n * g).abs() + y.abs()))), "z": (z, h * z.abs() + (1 + h) * bz),
           "m": (m, bm), "s": (s, s * (rel + 2 * E))}
    if dy is None:
        return res
    u, rows = dy * g, x.shape[0]
    c1, c2 = u.mean(-1, keepdim=True), (u * n).mean(-1, keepdim=True)
    b1 = 50 * E * u.abs().mean(-1, keepdim=True)
    b2 = 50 * E * (u * n).abs().mean(-1, keepdim=True) + (u.abs() * bn).mean(-1, keepdim=True)
    t = u - c1 - n * c2
    bt = 4 * E * (u.abs() + c1.abs() + (n * c2).abs()) + b1 + n.abs() * b2 + bn * c2.abs()
    dz, bdz = s * t, s * (bt + t.abs() * (rel + 3 * E))
    if dz_in is not None:
        dz = dz + dz_in
        bdz = bdz + E * (dz.abs() + dz_in.abs())
    fx = one if f is None else f
    dx = dz * fx
    # rows of one thread, the groups of a block and the blocks follow one another in the sum over the rows
    chain = (rows / 592 + 160) * E
    res.update({"dr": (dz, h * dz.abs() + (1 + h) * bdz), "dx": (dx, h * dx.abs() + (1 + h) * fx * (bdz + 2 * E * dz.abs())),
                "dgain": ((dy * n).sum(0), chain * (dy * n).abs().sum(0) + (dy.abs() * bn).sum(0) * 1.001),
                "dshift": (dy.sum(0), chain * dy.abs().sum(0))})
    return res
