"""Attention-based fusion of the ranking model's tokens with the graph encoder's states, and what its speed is judged by.

The feature tokens of a request (a candidate, a pair, the token stack of the fusion layer) attend to the encoder's
embeddings of a user's interaction sequence: queries and keys are normalised per head and rotated by their position in the
sequence, then every token takes the softmax-weighted mean of the sequence's values.  A case is one of these kinds:

  rotary    rotation of every head of a matrix by its row's position: half or interleaved pairs, part of the head, frequencies
            interpolated by parts for sequences beyond the trained length; `train` adds the gradient (the inverse rotation)
  qk_norm   root-mean-square norm of every head of queries and keys, with the rotation in the same pass; `train` adds the
            gradients with respect to the inputs and both gains
  attend    attention of ragged sequences of tokens to ragged sequences of states (fewer key heads than query heads where
            kv_heads < heads); `train` adds the gradients with respect to queries, keys and values

Sequences are ragged and packed: sequence s owns the rows q_ptr[s] .. q_ptr[s+1] of the queries and k_ptr[s] .. k_ptr[s+1]
of the keys.  The lengths go by the case, their order by the seed.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


# ------------------------------------------------------------------------------------------------- the cases

def _rotary(name, dtype, rows, heads, head_dim, rot, interleaved, far, factor, train):
    return dict(name=name, kind="rotary", dtype=dtype, rows=rows, heads=heads, head_dim=head_dim, rot=rot, interleaved=interleaved, far=far,
                factor=factor, train=train)


def _qk_norm(name, dtype, n_seq, max_q, max_k, heads, kv_heads, head_dim, rot, interleaved, train):
    return dict(name=name, kind="qk_norm", dtype=dtype, n_seq=n_seq, max_q=max_q, max_k=max_k, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                rot=rot, interleaved=interleaved, train=train)


def _attend(name, dtype, n_seq, max_q, max_k, heads, kv_heads, head_dim, masked, train):
    return dict(name=name, kind="attend", dtype=dtype, n_seq=n_seq, max_q=max_q, max_k=max_k, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                masked=masked, train=train)


def listed():
    return [
        # states of the large encoder (256 wide, four heads) of 65 536 history entries, rotated before they go into a cache
        _rotary("rotary_half_bf16", "bf16", 65_536, 4, 64, 64, False, 4_096, 1.0, False),
        # a check in fp32 with far positions (the event's minute), interleaved pairs, three quarters of a head, scaled frequencies
        _rotary("rotary_far_f32", "f32", 20_011, 2, 64, 48, True, 40_000_000, 8.0, True),
        # online inference for the 64 users of one request: one token each, histories of up to 100
        _qk_norm("qk_norm_serve_bf16", "bf16", 64, 1, 100, 4, 4, 32, 32, False, False),
        # the training step on 4096 pairs, medium width
        _qk_norm("qk_norm_train_bf16", "bf16", 4_096, 1, 100, 4, 4, 32, 32, False, True),
        # fp32 and odd sizes, fewer key heads than query heads, the rotation over half the head
        _qk_norm("qk_norm_ragged_f32", "f32", 333, 37, 211, 6, 2, 40, 20, True, True),
        # attention of the same 64 users: the smallest call, bound by latency
        _attend("attend_serve_bf16", "bf16", 64, 1, 100, 4, 4, 32, False, False),
        # single tokens over lifelong histories, four query heads per key head
        _attend("attend_long_bf16", "bf16", 4, 1, 32_768, 8, 2, 128, False, False),
        # a thousand candidates of each of four users scored against that user's history at once
        _attend("attend_candidates_bf16", "bf16", 4, 1_000, 4_096, 8, 4, 128, False, False),
        # the training step on 4096 pairs: one token each, histories of up to 100
        _attend("attend_pairs_train_bf16", "bf16", 4_096, 1, 100, 4, 4, 32, False, True),
        # the fusion layer itself: the stack of three tokens of 8192 requests attends to itself
        _attend("attend_tokens_train_bf16", "bf16", 8_192, 3, 3, 4, 4, 64, False, True),
        # the largest: batched sequences of tokens against padded histories whose padding the mask hides
        _attend("attend_train_bf16", "bf16", 8, 2_048, 4_096, 8, 8, 128, True, True),
        # a small experiment in fp32, ragged, heads of odd width
        _attend("attend_ragged_f32", "f32", 77, 61, 307, 4, 2, 36, True, True),
    ]


def _log(rng, lo, hi):
    return int(round(float(lo) * (float(hi) / lo) ** rng.random()))


def draw(rng):
    while True:
        c = _draw(rng)
        if _cost(c) <= 1.0 and _cost(c) > 1e-6:
            return c


def _draw(rng):
    kind = rng.choice(["rotary", "qk_norm", "qk_norm", "attend", "attend", "attend", "attend"])
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    train = rng.random() < 0.6
    head_dim = rng.choice([32, 64, 64, 128, 128, 16, 40, 80, 96] if dtype == "bf16" else [16, 32, 64, 64, 36, 100, 128])
    kv_heads = rng.choice([1, 2, 4, 4])
    heads = kv_heads * rng.choice([1, 1, 2, 4])
    rot = head_dim if rng.random() < 0.6 else 2 * rng.randint(1, head_dim // 2)
    interleaved = rng.random() < 0.5
    if kind == "rotary":
        c = _rotary("", dtype, _log(rng, 50, 200_000), heads, head_dim, rot, interleaved, _log(rng, 100, 100_000_000), rng.choice([1.0, 1.0, 4.0, 8.0]), train)
    else:
        n_seq = _log(rng, 1, 8_192)
        max_q = rng.choice([1, 1, 3, _log(rng, 2, 2_048), _log(rng, 2, 2_048)])
        max_k = rng.choice([100, 200, _log(rng, 1, 32_768), _log(rng, 16, 4_096)])
        if kind == "qk_norm":
            c = _qk_norm("", dtype, n_seq, max_q, max_k, heads, kv_heads, head_dim, rot, interleaved, train)
        else:
            c = _attend("", dtype, n_seq, max_q, max_k, heads, kv_heads, head_dim, rng.random() < 0.4, train)
    del c["name"]
    return c


def _cost(c):
    """A case's share of what the largest listed one takes: scores, and elements of queries and keys."""
    if c["kind"] == "rotary":
        return c["rows"] * c["heads"] * c["head_dim"] / 1.2e8
    rows = c["n_seq"] * (c["max_q"] * c["heads"] + 2 * c["max_k"] * c["kv_heads"]) * c["head_dim"]
    scores = c["n_seq"] * c["max_q"] * c["max_k"] * c["heads"] if c["kind"] == "attend" else 0
    return max(rows / 1.2e8, scores * (1 if c["dtype"] == "bf16" else 4) / (8.0 * 8 * 2_048 * 4_096))


# ------------------------------------------------------------------------------------------------- inputs

def _lengths(c):
    """Lengths of the sequences of a case, [n_seq, 2] (queries, keys): the first is as long as they get, some are empty."""
    n, r = c["n_seq"], np.random.default_rng([c["n_seq"], c["max_q"], c["max_k"]])

    def side(longest):
        v = r.integers(max(1, longest // 4), longest + 1, n)
        if n >= 32:
            v[r.integers(1, n, n // 32)] = 0
        v[0] = longest
        return v

    return np.stack([side(c["max_q"]), side(c["max_k"])], 1)


def _frequencies(rot, base=10_000.0, factor=1.0, trained=4_096.0, low=1.0, high=32.0):
    """Radians per position of every pair, float64.  With factor > 1 pairs that turn less than `low` times over the trained
    length are slowed down by it, pairs that turn more than `high` times are left alone, linearly in between."""
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    keep = ((trained * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
    return f * (keep + (1 - keep) / factor)


def prepare(case, seed):
    c, dt = case, DTYPES[case["dtype"]]
    gen = torch.Generator(device=DEV).manual_seed(int(seed))

    def normal(*shape, dtype=dt, mean=0.0):
        return (torch.randn(*shape, generator=gen, device=DEV) + mean).to(dtype)

    s = {"case": c}
    if c["kind"] == "rotary":
        w = c["heads"] * c["head_dim"]
        s["x"], s["freqs"] = normal(c["rows"], w), _frequencies(c["rot"], factor=c["factor"])
        s["pos"] = torch.randint(0, c["far"], (c["rows"],), generator=gen, device=DEV, dtype=torch.int32)
        s["mscale"] = 0.1 * math.log(c["factor"]) + 1.0          # the sharper softmax of stretched positions
        s["dy"] = normal(c["rows"], w) if c["train"] else None
        return s
    lens = torch.from_numpy(_lengths(c)).to(DEV)[torch.randperm(c["n_seq"], generator=gen, device=DEV)]
    ptr = torch.zeros(c["n_seq"] + 1, 2, dtype=torch.int64, device=DEV)
    ptr[1:] = lens.cumsum(0)
    s["q_ptr"], s["k_ptr"] = ptr[:, 0].contiguous(), ptr[:, 1].contiguous()
    nq, nk = (int(v) for v in _lengths(c).sum(0))
    wq, wk = c["heads"] * c["head_dim"], c["kv_heads"] * c["head_dim"]
    s["q"], s["k"] = normal(nq, wq), normal(nk, wk)
    if c["kind"] == "qk_norm":
        seq = torch.searchsorted(s["k_ptr"], torch.arange(nk, device=DEV), right=True) - 1
        s["pos_k"] = (torch.arange(nk, device=DEV) - s["k_ptr"][seq]).to(torch.int32)
        seq = torch.searchsorted(s["q_ptr"], torch.arange(nq, device=DEV), right=True) - 1
        s["pos_q"] = (lens[seq, 1] + torch.arange(nq, device=DEV) - s["q_ptr"][seq]).to(torch.int32)     # the tokens follow the history
        s["freqs"] = _frequencies(c["rot"])
        s["wq"], s["wk"] = 1 + 0.1 * normal(c["head_dim"], dtype=torch.float32), 1 + 0.1 * normal(c["head_dim"], dtype=torch.float32)
        if c["train"]:
            s["dqn"], s["dkn"] = normal(nq, wq), normal(nk, wk)
        return s
    s["v"], s["scale"] = normal(nk, wk, mean=0.25), c["head_dim"] ** -0.5
    s["mask"] = None
    if c["masked"]:       # a tail of padding behind each history, and single entries that a filter took out
        seq = torch.searchsorted(s["k_ptr"], torch.arange(nk, device=DEV), right=True) - 1
        at = (torch.arange(nk, device=DEV) - s["k_ptr"][seq]) / lens[seq, 1].clamp(min=1)
        tail = 0.75 + 0.25 * torch.rand(c["n_seq"], generator=gen, device=DEV)
        s["mask"] = ((at < tail[seq]) & (torch.rand(nk, generator=gen, device=DEV) > 0.02)).to(torch.uint8)
    s["dout"] = normal(nq, wq) if c["train"] else None
    return s


# ------------------------------------------------------------------------------------------------- plain forms

def _rotate(x, pos, freqs, interleaved, mscale, back=False):
    """x [rows, heads, head_dim] fp32, turned by pos * freqs (angles in 64 bits: far positions leave 32 no digits)."""
    r = 2 * freqs.numel()
    angle = pos.double()[:, None] * freqs
    cos, sin = (angle.cos() * mscale).float()[:, None], (angle.sin() * (-mscale if back else mscale)).float()[:, None]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., : r // 2], x[..., r // 2: r])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _heads(x, n):
    return x.float().view(x.shape[0], n, -1)


def _norm(x, w):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w


def _norm_back(g, x, w):
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n, gw = x * r, g * w
    return r * (gw - n * (gw * n).mean(-1, keepdim=True)), (g * n).double().sum((0, 1)).float()


def _plain_rotary(s):
    c = s["case"]
    y = _rotate(_heads(s["x"], c["heads"]), s["pos"], s["freqs"], c["interleaved"], s["mscale"])
    out = [y.flatten(1).to(s["x"].dtype)]
    if c["train"]:
        dx = _rotate(_heads(s["dy"], c["heads"]), s["pos"], s["freqs"], c["interleaved"], s["mscale"], back=True)
        out.append(dx.flatten(1).to(s["x"].dtype))
    return out


def _plain_qk_norm(s):
    c, dt = s["case"], s["q"].dtype
    q, k = _heads(s["q"], c["heads"]), _heads(s["k"], c["kv_heads"])
    out = [_rotate(_norm(q, s["wq"]), s["pos_q"], s["freqs"], c["interleaved"], 1.0).flatten(1).to(dt),
           _rotate(_norm(k, s["wk"]), s["pos_k"], s["freqs"], c["interleaved"], 1.0).flatten(1).to(dt)]
    if c["train"]:
        gq = _rotate(_heads(s["dqn"], c["heads"]), s["pos_q"], s["freqs"], c["interleaved"], 1.0, back=True)
        gk = _rotate(_heads(s["dkn"], c["kv_heads"]), s["pos_k"], s["freqs"], c["interleaved"], 1.0, back=True)
        (dq, dwq), (dk, dwk) = _norm_back(gq, q, s["wq"]), _norm_back(gk, k, s["wk"])
        out += [dq.flatten(1).to(dt), dk.flatten(1).to(dt), dwq, dwk]
    return out


def _padded(ptr, longest, rows):
    """Row of every place of a [n_seq, longest] batch, which places are in use, and the place of every row."""
    at = ptr[:-1, None] + torch.arange(longest, device=DEV)
    r = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(ptr, r, right=True) - 1
    return at.clamp(max=max(rows - 1, 0)), at < ptr[1:, None], seq * longest + r - ptr[seq]


def _plain_attend(s):
    c, dt = s["case"], s["q"].dtype
    H, G, hd, n = c["kv_heads"], c["heads"] // c["kv_heads"], c["head_dim"], c["n_seq"]
    qi, qu, qp = _padded(s["q_ptr"], c["max_q"], s["q"].shape[0])
    ki, ku, kp = _padded(s["k_ptr"], c["max_k"], s["k"].shape[0])
    if s["mask"] is not None:
        ku = ku & s["mask"][ki].bool()

    def tokens(x):        # [rows, heads * head_dim] -> [n, key head, query head of it * token, head_dim]
        return x[qi].float().view(n, -1, H, G, hd).permute(0, 2, 3, 1, 4).reshape(n, H, -1, hd)

    def states(x):
        return x[ki].float().view(n, -1, H, hd).transpose(1, 2)

    def packed(x):
        return x.view(n, H, G, -1, hd).permute(0, 3, 1, 2, 4).reshape(-1, H * G * hd)[qp].to(dt)

    q, k, v = tokens(s["q"]), states(s["k"]), states(s["v"])
    z = (q @ k.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(~ku[:, None, None], -math.inf)
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
        ds = (do @ v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
        dq, dk = ds @ k, ds.transpose(-1, -2) @ q
        out += [packed(dq)] + [x.transpose(1, 2).reshape(-1, H * hd)[kp].to(dt) for x in (dk, dv)]
    return out


# ------------------------------------------------------------------------------------------------- the calls of a user

def _own_rotary(s):
    import paper_2511_20564_b200 as E
    c = s["case"]
    out = [E.rotary(s["x"], c["heads"], s["freqs"], s["pos"], scale=s["mscale"], interleaved=c["interleaved"])]
    if c["train"]:
        out.append(E.rotary(s["dy"], c["heads"], s["freqs"], s["pos"], scale=s["mscale"], interleaved=c["interleaved"], inverse=True))
    return out


def _own_qk_norm(s):
    import paper_2511_20564_b200 as E
    c = s["case"]
    plan = dict(freqs=s["freqs"], pos_q=s["pos_q"], pos_k=s["pos_k"], eps=EPS, interleaved=c["interleaved"])
    out = list(E.qk_norm_rotary_forward(s["q"], s["k"], c["heads"], c["kv_heads"], s["wq"], s["wk"], **plan))
    if c["train"]:
        out += list(E.qk_norm_rotary_backward(s["dqn"], s["dkn"], s["q"], s["k"], c["heads"], c["kv_heads"], s["wq"], s["wk"], **plan))[:4]
    return out


def _own_attend(s):
    import paper_2511_20564_b200 as E
    c = s["case"]
    seqs = E.Sequences(s["q_ptr"], s["k_ptr"], max_q=c["max_q"], max_k=c["max_k"], k_mask=s["mask"])
    out, lse = E.cross_attention_forward(s["q"], s["k"], s["v"], seqs, c["heads"], c["kv_heads"], s["scale"])[:2]
    if not c["train"]:
        return [out, lse]
    return [out, lse] + list(E.cross_attention_backward(s["dout"], s["q"], s["k"], s["v"], out, lse, seqs, c["heads"], c["kv_heads"], s["scale"])[:3])


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"rotary": _own_rotary, "qk_norm": _own_qk_norm, "attend": _own_attend}[kind](state)
    return {"rotary": _plain_rotary, "qk_norm": _plain_qk_norm, "attend": _plain_attend}[kind](state)


# ------------------------------------------------------------------------------------------------- what a pass has to move

def work(case):
    c, es = case, 2 if case["dtype"] == "bf16" else 4
    hd = c["head_dim"]
    if c["kind"] == "rotary":
        n = c["rows"] * c["heads"]
        passes = 2 if c["train"] else 1
        return {"bytes": passes * (2 * n * hd * es + 4 * c["rows"]), "flops": passes * 3 * n * c["rot"]}
    lens = _lengths(c).astype(np.float64)
    nq, nk = (float(v) for v in lens.sum(0))
    q, k = nq * c["heads"] * hd, nk * c["kv_heads"] * hd
    if c["kind"] == "qk_norm":
        by, fl = 2 * (q + k) * es + 4 * (nq + nk), 7 * (q + k)
        if c["train"]:
            by, fl = by + 3 * (q + k) * es + 4 * (nq + nk), fl + 14 * (q + k)
        return {"bytes": by, "flops": fl}
    pairs = float((lens[:, 0] * lens[:, 1]).sum()) * c["heads"] * hd * (0.86 if c["masked"] else 1.0)
    by = (2 * q + 2 * k) * es + 4 * nq * c["heads"] + (nk if c["masked"] else 0) + 16 * c["n_seq"]
    if c["train"]:       # the tokens' and states' gradients, with everything read once more
        return {"bytes": by + (4 * q + 4 * k) * es, "flops": 14 * pairs}
    return {"bytes": by, "flops": 4 * pairs}


# ------------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    f64 = {name: v.double() for name, v in s.items() if isinstance(v, torch.Tensor)}
    return {"rotary": _exact_rotary, "qk_norm": _exact_qk_norm, "attend": _exact_attend}[case["kind"]](case, s, f64)


def _turned(x, heads, pos, freqs, interleaved, factor):
    """Every pair of a head as a complex number, multiplied by factor * exp(i angle)."""
    x = x.reshape(x.shape[0], heads, -1)
    y, half = x.clone(), freqs.numel()
    even = torch.arange(half, device=DEV) * (2 if interleaved else 1)
    odd = even + (1 if interleaved else half)
    turn = torch.polar(torch.full_like(pos[:, None] * freqs, abs(factor)), pos[:, None] * freqs)
    z = torch.complex(x[..., even], x[..., odd]) * (turn.conj() if factor < 0 else turn)[:, None]      # a negative factor turns back
    y[..., even], y[..., odd] = z.real, z.imag
    return y


def _exact_rotary(c, s, f):
    out = [_turned(f["x"], c["heads"], f["pos"], f["freqs"], c["interleaved"], s["mscale"]).flatten(1)]
    if c["train"]:
        out.append(_turned(f["dy"], c["heads"], f["pos"], f["freqs"], c["interleaved"], -s["mscale"]).flatten(1))
    return out


def _exact_qk_norm(c, s, f):
    made, grads, gains = [], [], []
    for x, w, pos, dy, heads in (("q", "wq", "pos_q", "dqn", c["heads"]), ("k", "wk", "pos_k", "dkn", c["kv_heads"])):
        h = f[x].reshape(-1, heads, c["head_dim"])
        rms = (h.square().sum(-1, keepdim=True) / c["head_dim"] + EPS).sqrt()
        made.append(_turned((h / rms * f[w]).flatten(1), heads, f[pos], f["freqs"], c["interleaved"], 1.0).flatten(1))
        if c["train"]:
            g = _turned(f[dy], heads, f[pos], f["freqs"], c["interleaved"], -1.0)
            inner = (g * f[w] * h).sum(-1, keepdim=True)
            grads.append((g * f[w] / rms - h * inner / (c["head_dim"] * rms ** 3)).flatten(1))
            gains.append((g * h / rms).sum((0, 1)))
    return made + grads + gains


def _exact_attend(c, s, f):
    H, G, hd = c["kv_heads"], c["heads"] // c["kv_heads"], c["head_dim"]
    out, lse = torch.zeros_like(f["q"]), torch.full((f["q"].shape[0], c["heads"]), -math.inf, dtype=torch.float64, device=DEV)
    dq, dk, dv = torch.zeros_like(f["q"]), torch.zeros_like(f["k"]), torch.zeros_like(f["v"])
    qp, kp = s["q_ptr"].tolist(), s["k_ptr"].tolist()
    for i in range(c["n_seq"]):
        rq = slice(qp[i], qp[i + 1])
        seen = torch.arange(kp[i], kp[i + 1], device=DEV)
        if s["mask"] is not None:
            seen = seen[s["mask"][seen] != 0]
        if rq.start == rq.stop or not seen.numel():
            continue
        q, k, v = f["q"][rq].view(-1, H, G, hd), f["k"][seen].view(-1, H, hd), f["v"][seen].view(-1, H, hd)
        z = torch.einsum("qhgd,khd->hgqk", q, k) * s["scale"]
        l = torch.logsumexp(z, -1)
        p = torch.exp(z - l[..., None])
        out[rq] = torch.einsum("hgqk,khd->qhgd", p, v).flatten(1)
        lse[rq] = l.permute(2, 0, 1).flatten(1)
        if c["train"]:
            do = f["dout"][rq].view(-1, H, G, hd)
            dv[seen] = torch.einsum("hgqk,qhgd->khd", p, do).flatten(1)
            dp = torch.einsum("qhgd,khd->hgqk", do, v)
            ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * s["scale"]
            dq[rq] = torch.einsum("hgqk,khd->qhgd", ds, k).flatten(1)
            dk[seen] = torch.einsum("hgqk,qhgd->khd", ds, q).flatten(1)
    return [out, lse] + ([dq, dk, dv] if c["train"] else [])
