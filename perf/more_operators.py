"""What stands around the attention of a fusion layer, and what its speed is judged by.

A layer of the ranking model lets its tokens attend to the encoder's states with a learned bias by the time that lies between them,
drops a share of what comes out while it trains, adds it to what went in and normalises the sum.  A case is one of these kinds:

  norm      layer norm of x, or of residual + dropout(x), with a gain and a shift; `keep_sum` also stores the sum (a layer that norms
            before it attends carries it on); `train` adds the gradients with respect to x, the residual, gain and shift
  dropout   dropout(x), or residual + dropout(x), from a counter-based generator; `train` adds the gradient, which forms the mask anew
  bias      attention of ragged sequences with a bias per head and bucket of the distance pos_k - pos_q; `train` adds the gradients with
            respect to queries, keys, values and the table of biases

Random numbers are inputs: a plan of a dropout is its rate, a seed, the number of the place and the step.  Element (row, col) is dropped
where its 16 bits of Philox4x32-10 with key seed and counter (col / 8, row, 2^31 + place, step) lie below round(p 2^16).  The bucket of a
pair is the number of edges that are not above its distance.  Sequences are ragged and packed as in the workloads of the attention.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


# ------------------------------------------------------------------------------------------------- the cases

def _norm(name, dtype, rows, dim, residual, p, keep_sum, train):
    return dict(name=name, kind="norm", dtype=dtype, rows=rows, dim=dim, residual=residual, p=p, keep_sum=keep_sum, train=train)


def _dropout(name, dtype, rows, dim, residual, p, train):
    return dict(name=name, kind="dropout", dtype=dtype, rows=rows, dim=dim, residual=residual, p=p, train=train)


def _bias(name, dtype, n_seq, max_q, max_k, heads, kv_heads, head_dim, order, buckets, far, both, masked, train):
    return dict(name=name, kind="bias", dtype=dtype, n_seq=n_seq, max_q=max_q, max_k=max_k, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                order=order, buckets=buckets, far=far, both=both, masked=masked, train=train)


def listed():
    return [
        # online inference for the 64 users of one request: one token each of the large encoder's width
        _norm("norm_serve_bf16", "bf16", 64, 256, True, 0.0, False, False),
        # the training step on 4096 pairs with histories of about 30 kept states: norm after the sum, dropout of the branch
        _norm("norm_train_bf16", "bf16", 131_072, 256, True, 0.1, False, True),
        # norm before the attention at the widest rows that the encoder takes: the sum goes on, its gradient comes back
        _norm("norm_stream_bf16", "bf16", 32_768, 1_024, True, 0.1, True, True),
        # a check in fp32 at the ranking tower's input width, odd rows, no residual
        _norm("norm_ragged_f32", "f32", 20_011, 320, False, 0.0, False, True),
        # dropout of the large encoder's states, forward and backward
        _dropout("dropout_train_bf16", "bf16", 262_144, 256, False, 0.1, True),
        # the hidden layer of the ranking tower in fp32, added to a residual
        _dropout("dropout_ragged_f32", "f32", 4_099, 516, True, 0.3, True),
        # the attention of the same 64 users with a bias by age: the smallest call, bound by latency
        _bias("bias_serve_bf16", "bf16", 64, 1, 100, 4, 4, 32, "after", 32, 100_000, False, False, False),
        # a thousand candidates of each of four users scored against that user's history at once
        _bias("bias_candidates_bf16", "bf16", 4, 1_000, 4_096, 8, 4, 128, "after", 32, 100_000, False, False, False),
        # the training step on 4096 pairs: one token each, histories of up to 100
        _bias("bias_pairs_train_bf16", "bf16", 4_096, 1, 100, 4, 4, 32, "after", 32, 100_000, False, False, True),
        # the largest: histories attend to themselves, both directions of time, padding hidden
        _bias("bias_train_bf16", "bf16", 8, 2_048, 2_048, 8, 8, 128, "self", 32, 20_000, True, True, True),
        # a small experiment in fp32, ragged, heads of odd width, distances by row number
        _bias("bias_ragged_f32", "f32", 77, 61, 307, 4, 2, 36, "index", 16, 128, True, True, True),
    ]


def _log(rng, lo, hi):
    return int(round(float(lo) * (float(hi) / lo) ** rng.random()))


def draw(rng):
    while True:
        c = _draw(rng)
        if 1e-6 < _cost(c) <= 1.0:
            del c["name"]
            return c


def _draw(rng):
    kind = rng.choice(["norm", "norm", "dropout", "bias", "bias", "bias"])
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    train = rng.random() < 0.7
    if kind != "bias":
        rows, dim = _log(rng, 1, 300_000), 8 * _log(rng, 1, 512) if dtype == "bf16" else 4 * _log(rng, 2, 512)
        p = rng.choice([0.1, 0.2, 0.5, round(rng.random() * 0.9, 3)])
        residual = rng.random() < 0.6
        if kind == "dropout":
            return _dropout("", dtype, rows, dim, residual, p, train)
        return _norm("", dtype, rows, dim, residual, p if rng.random() < 0.6 else 0.0, residual and rng.random() < 0.5, train)
    head_dim = rng.choice([32, 64, 64, 128, 128, 16, 40, 80, 96] if dtype == "bf16" else [16, 32, 64, 64, 36, 100, 128])
    kv_heads = rng.choice([1, 2, 4, 4])
    heads = kv_heads * rng.choice([1, 1, 2, 4])
    n_seq = _log(rng, 1, 4_096)
    max_q = rng.choice([1, 1, 3, _log(rng, 2, 2_048), _log(rng, 2, 2_048)])
    max_k = rng.choice([100, 200, _log(rng, 1, 16_384), _log(rng, 16, 4_096)])
    order = rng.choice(["after", "after", "index", "self"])
    if order == "self":
        max_k = max_q = max(max_q, 2)
    return _bias("", dtype, n_seq, max_q, max_k, heads, kv_heads, head_dim, order, rng.randint(2, 60), _log(rng, 64, 1_000_000), rng.random() < 0.5,
                 rng.random() < 0.4, train)


def _cost(c):
    """A case's share of what the largest listed one of its kind takes: elements, or scores and elements of queries and keys."""
    if c["kind"] == "norm":
        return c["rows"] * c["dim"] / (131_072 * 256) * (1 if c["dtype"] == "bf16" else 2)
    if c["kind"] == "dropout":
        return c["rows"] * c["dim"] / (262_144 * 256) * (1 if c["dtype"] == "bf16" else 2)
    rows = c["n_seq"] * (c["max_q"] * c["heads"] + 2 * c["max_k"] * c["kv_heads"]) * c["head_dim"]
    scores = c["n_seq"] * c["max_q"] * c["max_k"] * c["heads"]
    return max(rows / 1.2e8, scores * (1 if c["dtype"] == "bf16" else 4) / (8.0 * 8 * 2_048 * 2_048))


# ------------------------------------------------------------------------------------------------- inputs

def _lengths(c):
    """Lengths of the sequences of a case, [n_seq, 2] (queries, keys): the first is as long as they get, some are empty."""
    n, r = c["n_seq"], np.random.default_rng([c["n_seq"], c["max_q"], c["max_k"], 5])

    def side(longest):
        v = r.integers(max(1, longest // 4), longest + 1, n)
        if n >= 32:
            v[r.integers(1, n, n // 32)] = 0
        v[0] = longest
        return v

    q, k = side(c["max_q"]), side(c["max_k"])
    return np.stack([k if c["order"] == "self" else q, k], 1)


def _edges(buckets, far, both):
    """Ascending edges of buckets by distance: bucket number by number up to half of them, then evenly by the logarithm up to `far`,
    on the side of the past and, with `both`, the same widths on the side of the future."""
    half, first = max(buckets // 2, 1), []
    for n in range(1, buckets):
        t = float(n) if n < half else half * (max(far, half + 1) / half) ** ((n - half) / max(buckets - half, 1))
        whole = round(t)
        t = whole if abs(t - whole) < 1e-9 * t else math.ceil(t)
        first.append(max(t, first[-1] + 1 if first else 1))
    return [1 - t for t in reversed(first)] + (first if both else [])


def prepare(case, seed):
    c, dt = case, DTYPES[case["dtype"]]
    gen = torch.Generator(device=DEV).manual_seed(int(seed))

    def normal(*shape, dtype=dt, mean=0.0, spread=1.0):
        return (torch.randn(*shape, generator=gen, device=DEV) * spread + mean).to(dtype)

    s = {"case": c}
    if c["kind"] != "bias":
        shape = (c["rows"], c["dim"])
        s["x"] = normal(*shape, mean=0.1)
        s["residual"] = normal(*shape, spread=1.5) if c["residual"] else None
        s["drop"] = dict(p=c["p"], seed=(int(seed) * 0x9E3779B97F4A7C15 + 12_345) % 2 ** 64, place=3, step=int(seed) % 1_000)
        s["dy"] = normal(*shape) if c["train"] else None
        if c["kind"] == "norm":
            s["gain"], s["shift"] = normal(c["dim"], dtype=torch.float32, mean=1.0, spread=0.1), normal(c["dim"], dtype=torch.float32, spread=0.1)
            s["dz"] = normal(*shape) if c["train"] and c["keep_sum"] else None
        return s
    lens = torch.from_numpy(_lengths(c)).to(DEV)[torch.randperm(c["n_seq"], generator=gen, device=DEV)]
    ptr = torch.zeros(c["n_seq"] + 1, 2, dtype=torch.int64, device=DEV)
    ptr[1:] = lens.cumsum(0)
    s["q_ptr"], s["k_ptr"] = ptr[:, 0].contiguous(), ptr[:, 1].contiguous()
    nq, nk = (int(v) for v in _lengths(c).sum(0))
    wq, wk = c["heads"] * c["head_dim"], c["kv_heads"] * c["head_dim"]
    s["q"], s["k"], s["v"], s["scale"] = normal(nq, wq), normal(nk, wk), normal(nk, wk, mean=0.25), c["head_dim"] ** -0.5
    s["pos_q"] = s["pos_k"] = None
    if c["order"] != "index":        # minutes at which the entries of a history came, and the tokens after it (or the entries themselves)
        gaps = (torch.rand(nk, generator=gen, device=DEV).clamp(min=1e-6).log() * -20).long()
        times = gaps.cumsum(0)
        seq = torch.searchsorted(s["k_ptr"], torch.arange(nk, device=DEV), right=True) - 1
        times = torch.cat([times, times.new_zeros(1)])
        begin = times[s["k_ptr"][:-1].clamp(max=max(nk - 1, 0))]
        s["pos_k"] = (times[:nk] - begin[seq]).to(torch.int32)
        if c["order"] == "self":
            s["pos_q"] = s["pos_k"].clone()
        else:
            seq = torch.searchsorted(s["q_ptr"], torch.arange(nq, device=DEV), right=True) - 1
            last = times[(s["k_ptr"][1:] - 1).clamp(min=0)] - begin
            s["pos_q"] = (torch.where(lens[:, 1] > 0, last, torch.zeros_like(last))[seq] + 1 + torch.arange(nq, device=DEV) - s["q_ptr"][seq]).to(torch.int32)
    s["edges"] = torch.tensor(_edges(c["buckets"], c["far"], c["both"]), dtype=torch.int32, device=DEV)
    s["table"] = normal(s["edges"].numel() + 1, c["heads"], dtype=torch.float32)
    s["mask"] = None
    if c["masked"]:       # a tail of padding behind each history, and single entries that a filter took out
        seq = torch.searchsorted(s["k_ptr"], torch.arange(nk, device=DEV), right=True) - 1
        at = (torch.arange(nk, device=DEV) - s["k_ptr"][seq]) / lens[seq, 1].clamp(min=1)
        tail = 0.75 + 0.25 * torch.rand(c["n_seq"], generator=gen, device=DEV)
        s["mask"] = ((at < tail[seq]) & (torch.rand(nk, generator=gen, device=DEV) > 0.02)).to(torch.uint8)
    s["dout"] = normal(nq, wq) if c["train"] else None
    return s


# ------------------------------------------------------------------------------------------------- plain forms

def _philox(counter, key):
    """Ten rounds on four 32-bit words held in int64 tensors (products wrap: their low 64 bits are what is wanted)."""
    low = 0xFFFFFFFF
    c0, c1, c2, c3 = counter
    k0, k1 = key
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _threshold(p):
    return min(int(math.floor(p * 65_536 + 0.5)), 65_535)


def _kept(drop, rows, dim):
    """Which elements of a [rows, dim] matrix stay."""
    unit, row = torch.arange((dim + 7) // 8, device=DEV), torch.arange(rows, device=DEV)
    shape = (rows, unit.numel())
    words = _philox((unit.expand(shape), row[:, None].expand(shape), torch.full(shape, 2 ** 31 + drop["place"], device=DEV),
                     torch.full(shape, drop["step"], device=DEV)), (drop["seed"] & 0xFFFFFFFF, drop["seed"] >> 32))
    bits = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], -1).view(rows, -1)[:, :dim]
    return bits >= _threshold(drop["p"])


def _dropped(x, drop, kept):
    t = _threshold(drop["p"])
    return x.float() if t == 0 else torch.where(kept, x.float() * (65_536.0 / (65_536 - t)), 0.0)


def _plain_dropout(s):
    dt, kept = s["x"].dtype, _kept(s["drop"], *s["x"].shape)
    y = _dropped(s["x"], s["drop"], kept)
    out = [(y if s["residual"] is None else s["residual"].float() + y).to(dt)]
    if s["dy"] is not None:
        out.append(_dropped(s["dy"], s["drop"], kept).to(dt))
    return out


def _plain_norm(s):
    c, dt = s["case"], s["x"].dtype
    kept = _kept(s["drop"], c["rows"], c["dim"]) if c["p"] else None
    z = _dropped(s["x"], s["drop"], kept)
    z = z if s["residual"] is None else s["residual"].float() + z
    mean = z.mean(-1, keepdim=True)
    n = z - mean
    r = torch.rsqrt((n * n).mean(-1, keepdim=True) + EPS)
    n = n * r
    out = [(n * s["gain"] + s["shift"]).to(dt)]
    if c["keep_sum"]:
        out.append(z.to(dt))
    if c["train"]:
        dy = s["dy"].float()
        g = dy * s["gain"]
        dz = r * (g - g.mean(-1, keepdim=True) - n * (g * n).mean(-1, keepdim=True))
        dz = dz if s["dz"] is None else dz + s["dz"].float()
        out.append(_dropped(dz, s["drop"], kept).to(dt))
        if s["residual"] is not None:
            out.append(dz.to(dt))
        out += [(dy * n).sum(0, dtype=torch.float64).float(), dy.sum(0, dtype=torch.float64).float()]
    return out


def _padded(ptr, longest, rows):
    """Row of every place of a [n_seq, longest] batch, which places are in use, and the place of every row."""
    at = ptr[:-1, None] + torch.arange(longest, device=DEV)
    r = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(ptr, r, right=True) - 1
    return at.clamp(max=max(rows - 1, 0)), at < ptr[1:, None], seq * longest + r - ptr[seq]


def _plain_bias(s):
    c, dt = s["case"], s["q"].dtype
    H, G, hd, n = c["kv_heads"], c["heads"] // c["kv_heads"], c["head_dim"], c["n_seq"]
    longest_q = c["max_k"] if c["order"] == "self" else c["max_q"]
    qi, qu, qp = _padded(s["q_ptr"], longest_q, s["q"].shape[0])
    ki, ku, kp = _padded(s["k_ptr"], c["max_k"], s["k"].shape[0])
    if s["mask"] is not None:
        ku = ku & s["mask"][ki].bool()
    if s["pos_q"] is None:
        pq, pk = torch.arange(longest_q, device=DEV).expand(n, -1), torch.arange(c["max_k"], device=DEV).expand(n, -1)
    else:
        pq, pk = s["pos_q"][qi].long(), s["pos_k"][ki].long()
    bucket = torch.searchsorted(s["edges"].long(), (pk[:, None] - pq[:, :, None]).contiguous(), right=True).to(torch.int32)

    def tokens(x):        # [rows, heads * head_dim] -> [n, key head, query head of it * token, head_dim]
        return x[qi].float().view(n, -1, H, G, hd).permute(0, 2, 3, 1, 4).reshape(n, H, -1, hd)

    def states(x):
        return x[ki].float().view(n, -1, H, hd).transpose(1, 2)

    def packed(x):
        return x.view(n, H, G, -1, hd).permute(0, 3, 1, 2, 4).reshape(-1, H * G * hd)[qp].to(dt)

    q, k, v = tokens(s["q"]), states(s["k"]), states(s["v"])
    z = (q @ k.transpose(-1, -2)).mul_(s["scale"])
    heads = z.view(n, H, G, longest_q, -1)
    for h in range(H * G):
        heads[:, h // G, h % G] += s["table"][:, h][bucket]
    z = z.masked_fill_(~ku[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total == 0, torch.ones_like(total), total))
    o = p @ v
    lse = (top + total.log()).view(n, H, G, -1).permute(0, 3, 1, 2).reshape(-1, H * G)[qp]
    out = [packed(o), lse]
    if c["train"]:
        do = (tokens(s["dout"]).view(n, H, G, -1, hd) * qu[:, None, None, :, None]).view(n, H, -1, hd)
        dv = p.transpose(-1, -2) @ do
        ds = (do @ v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p)
        dtable = torch.zeros(s["table"].shape, dtype=torch.float64, device=DEV)
        whole = ds.view(n, H * G, longest_q, -1)
        for b in torch.unique(bucket).tolist():
            dtable[b] = (whole * (bucket == b)[:, None]).sum(-1).sum((0, 2), dtype=torch.float64)
        ds = ds.mul_(s["scale"])
        dq, dk = ds @ k, ds.transpose(-1, -2) @ q
        out += [packed(dq)] + [x.transpose(1, 2).reshape(-1, H * hd)[kp].to(dt) for x in (dk, dv)] + [dtable.float()]
    return out


# ------------------------------------------------------------------------------------------------- the calls of a user

def _own_plan(s):
    import paper_2511_20564_b200 as E
    d = s["drop"]
    return E.Dropout(d["p"], d["seed"], place=d["place"], step=d["step"]) if d["p"] else None


def _own_dropout(s):
    import paper_2511_20564_b200 as E
    plan = _own_plan(s)
    out = [E.dropout(s["x"], plan, residual=s["residual"])]
    if s["dy"] is not None:
        out.append(E.dropout(s["dy"], plan))
    return out


def _own_norm(s):
    import paper_2511_20564_b200 as E
    c, plan = s["case"], _own_plan(s)
    y, z, stats = E.layer_norm_forward(s["x"], s["gain"], s["shift"], residual=s["residual"], drop=plan, eps=EPS, keep_sum=c["keep_sum"],
                                       keep_stats=c["train"])
    out = [y, z] if c["keep_sum"] else [y]
    if c["train"]:
        dx, dr, dgain, dshift, _ = E.layer_norm_backward(s["dy"], s["x"], stats, s["gain"], residual=s["residual"], drop=plan, dZ=s["dz"])
        out += [dx, dgain, dshift] if s["residual"] is None else [dx, dr, dgain, dshift]
    return out


def _own_bias(s):
    import paper_2511_20564_b200 as E
    c = s["case"]
    longest_q = c["max_k"] if c["order"] == "self" else c["max_q"]
    seqs = E.Sequences(s["q_ptr"], s["k_ptr"], max_q=longest_q, max_k=c["max_k"], k_mask=s["mask"])
    bias = E.RelativeBias(s["table"], s["edges"], pos_q=s["pos_q"], pos_k=s["pos_k"])
    out, lse = E.biased_attention_forward(s["q"], s["k"], s["v"], seqs, bias, c["heads"], c["kv_heads"], s["scale"])[:2]
    if not c["train"]:
        return [out, lse]
    return [out, lse] + list(E.biased_attention_backward(s["dout"], s["q"], s["k"], s["v"], out, lse, seqs, bias, c["heads"], c["kv_heads"],
                                                         s["scale"])[:4])


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"norm": _own_norm, "dropout": _own_dropout, "bias": _own_bias}[kind](state)
    return {"norm": _plain_norm, "dropout": _plain_dropout, "bias": _plain_bias}[kind](state)


# ------------------------------------------------------------------------------------------------- what a pass has to move

def work(case):
    c, es = case, 2 if case["dtype"] == "bf16" else 4
    if c["kind"] != "bias":
        n, r = c["rows"] * c["dim"], int(c["residual"])
        matrices = 2 + r                                                     # x, residual -> y
        if c["kind"] == "norm":
            matrices += int(c["keep_sum"])
        if c["train"]:
            if c["kind"] == "dropout":
                matrices += 2                                                # dy -> dx
            else:                                                            # dy, x, residual, dz -> dx, and dr where it is another
                matrices += 3 + r + int(c["keep_sum"]) + int(bool(r and c["p"]))
        flops = n * ((8 if c["kind"] == "norm" else 1) * (1 + 2 * int(c["train"])))
        return {"bytes": matrices * n * es, "flops": flops}
    lens = _lengths(c).astype(np.float64)
    nq, nk = (float(v) for v in lens.sum(0))
    q, k = nq * c["heads"] * c["head_dim"], nk * c["kv_heads"] * c["head_dim"]
    pairs = float((lens[:, 0] * lens[:, 1]).sum()) * c["heads"] * c["head_dim"] * (0.86 if c["masked"] else 1.0)
    by = (2 * q + 2 * k) * es + 4 * nq * c["heads"] + (nk if c["masked"] else 0) + 16 * c["n_seq"] + (0 if c["order"] == "index" else 4 * (nq + nk))
    if c["train"]:       # the tokens' and states' gradients, with everything read once more
        return {"bytes": by + (4 * q + 4 * k) * es, "flops": 14 * pairs}
    return {"bytes": by, "flops": 4 * pairs}


# ------------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    f64 = {name: v.double() for name, v in s.items() if isinstance(v, torch.Tensor)}
    return {"norm": _exact_norm, "dropout": _exact_dropout, "bias": _exact_bias}[case["kind"]](case, s, f64)


def _factors(drop, rows, dim):
    """What every element is multiplied by: 0, or one over the share that stays.  Unsigned 64-bit words on the host."""
    cut = min(int(math.floor(drop["p"] * 2.0 ** 16 + 0.5)), 2 ** 16 - 1)
    units = -(-dim // 8)
    words = np.empty((4, rows, units), dtype=np.uint64)
    words[0], words[1] = np.arange(units, dtype=np.uint64), np.arange(rows, dtype=np.uint64)[:, None]
    words[2], words[3] = 2 ** 31 + drop["place"], drop["step"]
    low, shift = np.uint64(2 ** 32 - 1), np.uint64(32)
    for i in range(10):
        keys = [np.uint64((drop["seed"] % 2 ** 32 + i * 0x9E3779B9) % 2 ** 32), np.uint64((drop["seed"] // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32)]
        even, odd = words[0] * np.uint64(0xD2511F53), words[2] * np.uint64(0xCD9E8D57)
        words = np.stack([(odd >> shift) ^ words[1] ^ keys[0], odd & low, (even >> shift) ^ words[3] ^ keys[1], even & low])
    halves = words.transpose(1, 2, 0).astype(np.uint32).copy().view(np.uint16).reshape(rows, units * 8)[:, :dim]
    return torch.from_numpy(np.where(halves < cut, 0.0, 2.0 ** 16 / (2 ** 16 - cut))).to(DEV)


def _exact_dropout(c, s, f):
    factor = _factors(s["drop"], c["rows"], c["dim"])
    out = [torch.addcmul(f["residual"], f["x"], factor) if c["residual"] else f["x"] * factor]
    return out + ([f["dy"] * factor] if c["train"] else [])


def _exact_norm(c, s, f):
    factor = _factors(s["drop"], c["rows"], c["dim"]) if c["p"] else 1.0
    z = f["x"] * factor + (f["residual"] if c["residual"] else 0.0)
    var, mean = torch.var_mean(z, -1, correction=0, keepdim=True)
    sd = (var + EPS).sqrt()
    out = [(z - mean) / sd * f["gain"] + f["shift"]] + ([z] if c["keep_sum"] else [])
    if c["train"]:
        g = f["dy"] * f["gain"]
        inner = (g * (z - mean)).sum(-1, keepdim=True)
        dz = (g - g.sum(-1, keepdim=True) / c["dim"]) / sd - (z - mean) * inner / (c["dim"] * sd ** 3)
        if c["keep_sum"]:
            dz = dz + f["dz"]
        out += [dz * factor] + ([dz] if c["residual"] else []) + [((z - mean) / sd * f["dy"]).sum(0), f["dy"].sum(0)]
    return out


def _exact_bias(c, s, f):
    H, G, hd = c["kv_heads"], c["heads"] // c["kv_heads"], c["head_dim"]
    out, lse = torch.zeros_like(f["q"]), torch.full((f["q"].shape[0], c["heads"]), -math.inf, dtype=torch.float64, device=DEV)
    dq, dk, dv, dtable = (torch.zeros_like(f[x]) for x in ("q", "k", "v", "table"))
    qp, kp, numbers = s["q_ptr"].tolist(), s["k_ptr"].tolist(), torch.arange(s["table"].shape[0], device=DEV)
    edges = s["edges"].long()
    for i in range(c["n_seq"]):
        rq = slice(qp[i], qp[i + 1])
        seen = torch.arange(kp[i], kp[i + 1], device=DEV)
        if s["mask"] is not None:
            seen = seen[s["mask"][seen] != 0]
        if rq.start == rq.stop or not seen.numel():
            continue
        if s["pos_q"] is None:
            apart = (seen - kp[i])[None] - torch.arange(rq.stop - rq.start, device=DEV)[:, None]
        else:
            apart = s["pos_k"][seen].long()[None] - s["pos_q"][rq].long()[:, None]
        bucket = torch.zeros_like(apart)
        for e in edges if apart.numel() > 2 ** 20 else ():
            bucket += apart >= e
        if apart.numel() <= 2 ** 20:
            bucket = (apart[..., None] >= edges).sum(-1)
        q, k, v = f["q"][rq].view(-1, H, G, hd), f["k"][seen].view(-1, H, hd), f["v"][seen].view(-1, H, hd)
        z = torch.einsum("qhgd,khd->hgqk", q, k) * s["scale"] + f["table"][bucket].permute(2, 0, 1).view(H, G, *bucket.shape)
        l = torch.logsumexp(z, -1)
        p = torch.exp(z - l[..., None])
        out[rq] = torch.einsum("hgqk,khd->qhgd", p, v).flatten(1)
        lse[rq] = l.permute(2, 0, 1).flatten(1)
        if c["train"]:
            do = f["dout"][rq].view(-1, H, G, hd)
            dv[seen] = torch.einsum("hgqk,qhgd->khd", p, do).flatten(1)
            dp = torch.einsum("qhgd,khd->hgqk", do, v)
            ds = p * (dp - (p * dp).sum(-1, keepdim=True))
            dq[rq] = torch.einsum("hgqk,khd->qhgd", ds, k).flatten(1) * s["scale"]
            dk[seen] = torch.einsum("hgqk,qhgd->khd", ds, q).flatten(1) * s["scale"]
            step = max(1, 2 ** 27 // (bucket.shape[1] * numbers.numel()))
            for a in range(0, bucket.shape[0], step):        # which bucket a pair is in as a matrix of zeros and ones
                which = (bucket[a: a + step].reshape(-1, 1) == numbers).double()
                dtable += which.T @ ds[:, :, a: a + step].reshape(H * G, -1).T
    return [out, lse] + ([dq, dk, dv, dtable] if c["train"] else [])
