"""Rotary positions and norms of queries and keys with the rotation, against their 64-bit form."""
import pytest
import torch

import fusion_oracle as F

pytestmark = pytest.mark.gpu

E24 = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


def _randn(*shape, seed, dtype):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def _held(got, want, bound, what):
    err = (got.double().cpu() - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), (err / bound).max().item())


def _trig(dtype):
    # sine and cosine: the hardware's of the reduced angle for 16-bit results (2^-20 with the reduction's rounding), series of five
    # terms in 32 bits for 32-bit ones (some four roundings of 2^-24 and 2^-25 of truncation); products and their sum add two roundings
    return 2.0 ** -20 if dtype == BF16 else 2.0 ** -21


SHAPES = [                                   # rows, heads, head_dim, rot, interleaved
    (1, 1, 8, 8, False), (3, 4, 32, 32, False), (257, 2, 64, 64, True), (130, 3, 40, 40, False), (77, 5, 40, 20, True),
    (65, 2, 128, 38, False), (33, 1, 256, 256, False), (19, 7, 96, 0, False), (300, 2, 16, 2, False), (41, 9, 80, 80, True),
    (29, 2, 128, 100, False), (1001, 1, 128, 128, False), (12, 33, 64, 48, True)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,hd,rot,inter", SHAPES)
def test_rotary_and_its_inverse(rows, heads, hd, rot, inter, dtype):
    import paper_2511_20564_b200 as E
    x = _randn(rows, heads * hd, seed=rows, dtype=dtype)
    pos = torch.randint(-(1 << 31), 1 << 31, (rows,), generator=torch.Generator().manual_seed(1), dtype=torch.int64)
    pos[::3] = torch.arange(rows)[::3]
    f = F.frequencies(rot) if rot else torch.empty(0, dtype=torch.float64)
    fd, pd = (f.cuda() if rot else None), pos.to(torch.int32).cuda()
    bound = lambda want, s: F.HALF[dtype] * want.abs() + (_trig(dtype) + 4 * E24) * F.rotate_scale(x.double(), heads, f, s, inter) + 2.0 ** -126
    for inverse in (False, True):
        want = F.rotate(x.double(), heads, f, pos, 1.25, inter, inverse)
        got = E.rotary(x.cuda(), heads, fd, pd, scale=1.25, interleaved=inter, inverse=inverse)
        _held(got, want, bound(want, 1.25), ("rotary", inverse))
    # in place, positions = row numbers
    y = x.cuda()
    assert E.rotary(y, heads, fd, None, interleaved=inter, out=y) is y
    want = F.rotate(x.double(), heads, f, torch.arange(rows), 1.0, inter)
    _held(y, want, bound(want, 1.0), "in place")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_rotary_of_a_column_range_leaves_its_neighbours(dtype):
    import paper_2511_20564_b200 as E
    wide = _randn(50, 5 * 64, seed=9, dtype=dtype).cuda()
    before, f = wide.clone(), F.frequencies(64).cuda()
    part = wide[:, 64:192]
    E.rotary(part, 2, f, None, out=part)
    assert torch.equal(wide[:, :64], before[:, :64]) and torch.equal(wide[:, 192:], before[:, 192:])
    assert torch.equal(part, E.rotary(before[:, 64:192].contiguous(), 2, f, None))


def test_frequencies():
    import paper_2511_20564_b200 as E
    for rot, base, factor, trained in ((64, 1e4, 1.0, 0.0), (48, 5e5, 8.0, 4096.0), (2, 1e4, 2.0, 128.0)):
        got = E.rotary_frequencies(rot, base, factor, trained).cpu()
        assert torch.allclose(got, F.frequencies(rot, base, factor, trained), rtol=1e-14, atol=0)     # pow: a few steps of 2^-52


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,hd,rot,inter", SHAPES)
def test_qk_norm_forward_and_backward(rows, heads, hd, rot, inter, dtype):
    """Queries and keys of different row counts and heads in one call; one row is all zeros (its norm rests on eps alone)."""
    import paper_2511_20564_b200 as E
    kv = max(1, heads // 2)
    k_rows = 2 * rows + 5
    q, k = _randn(rows, heads * hd, seed=2, dtype=dtype), _randn(k_rows, kv * hd, seed=3, dtype=dtype)
    k[1] = 0
    dq, dk = _randn(rows, heads * hd, seed=4, dtype=dtype), _randn(k_rows, kv * hd, seed=5, dtype=dtype)
    wq, wk = 1 + 0.2 * _randn(hd, seed=6, dtype=F32), 1 + 0.2 * _randn(hd, seed=7, dtype=F32)
    pq, pk = torch.arange(rows, dtype=torch.int32) + 1000, torch.arange(k_rows, dtype=torch.int32)
    f = F.frequencies(rot) if rot else torch.empty(0, dtype=torch.float64)
    plan = dict(freqs=f.cuda() if rot else None, pos_q=pq.cuda(), pos_k=pk.cuda(), eps=1e-5, scale=1.0, interleaved=inter)
    cu = lambda *ts: [t.cuda() for t in ts]
    qn, kn = E.qk_norm_rotary_forward(*cu(q, k), heads, kv, *cu(wq, wk), **plan)
    got = E.qk_norm_rotary_backward(*cu(dq, dk, q, k), heads, kv, *cu(wq, wk), **plan)
    again = E.qk_norm_rotary_backward(*cu(dq, dk, q, k), heads, kv, *cu(wq, wk), **plan)
    for i in range(4):
        assert torch.equal(got[i], again[i])
    norm = (hd + 8) * E24             # relative error of 1 / rms and of a mean over a head in 32 bits
    for i, (x, g, w, n, pos, y) in enumerate(((q, dq, wq, heads, pq, qn), (k, dk, wk, kv, pk, kn))):
        x, g, w, pos = x.double(), g.double(), w.double(), pos.long()
        h = F.norm(x, n, w, 1e-5)
        want = F.rotate(h, n, f, pos, 1.0, inter)
        _held(y, want, F.HALF[dtype] * want.abs() + (_trig(dtype) + norm) * F.rotate_scale(h, n, f, 1.0, inter) + 2.0 ** -126, "forward")
        dx, dw, dx_terms, dw_terms = F.norm_rotary_backward(g, x, n, w, 1e-5, f, pos, 1.0, inter)
        _held(got[i], dx, F.HALF[dtype] * dx.abs() + (_trig(dtype) + 3 * norm) * dx_terms + 2.0 ** -126, "dx")
        # no chain of additions is longer than the terms of one thread, 8 warps and all blocks' partial sums
        _held(got[2 + i], dw, (_trig(dtype) + 3 * norm + (x.shape[0] * n + 600) * E24) * dw_terms, "dw")


def test_qk_norm_without_gains_keys_or_rows():
    import paper_2511_20564_b200 as E
    x = _randn(10, 64, seed=1, dtype=F32).cuda()
    y, none = E.qk_norm_rotary_forward(x, None, 2, 1)
    want = F.norm(x.double().cpu(), 2, torch.ones(32, dtype=torch.float64), 1e-6)
    assert none is None
    _held(y, want, 64 * E24 * want.abs(), "norm alone")
    dx, dk, dw, dwk, _ = E.qk_norm_rotary_backward(x, None, x, None, 2, 1)
    assert dk is None and dwk is None and dw.shape == (32,)
    dx2, _, dw2, _, _ = E.qk_norm_rotary_backward(x, None, x, None, 2, 1, gains=False)
    assert dw2 is None and torch.equal(dx, dx2)
    empty = x[:0]
    dx, _, dw, _, _ = E.qk_norm_rotary_backward(empty, None, empty, None, 2, 1)
    assert dx.shape == (0, 64) and not dw.any()
    assert E.rotary(empty, 2, None).shape == (0, 64)


def test_many_rows_of_gains():
    """Gains summed over more rows than one turn of all blocks takes."""
    import paper_2511_20564_b200 as E
    rows, heads, hd = 200_003, 2, 32
    x = torch.randn(rows, heads * hd, generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(BF16)
    g = torch.randn(rows, heads * hd, generator=torch.Generator("cuda").manual_seed(2), device="cuda").to(BF16)
    dx, _, dw, _, _ = E.qk_norm_rotary_backward(g, None, x, None, heads, 1)
    h = x.double().view(rows, heads, hd)
    n = h / (h.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    terms = g.double().view(rows, heads, hd) * n
    assert ((dw - terms.sum((0, 1))).abs() <= (rows * heads / (148 * 4) + 700) * E24 * terms.abs().sum((0, 1))).all()


def test_wrong_matrices_are_errors():
    import paper_2511_20564_b200 as E
    x, line, half = torch.zeros(4, 64, device="cuda"), torch.zeros(64, device="cuda"), torch.zeros(4, 64, device="cuda", dtype=torch.float16)
    ptr = torch.tensor([0, 4], device="cuda")
    seqs = E.Sequences(ptr, ptr)
    lse = torch.zeros(4, 2, device="cuda")
    for bad in (line, half, x.cpu(), x.t(), None):
        for call in (lambda: E.qk_norm_rotary_backward(bad, None, x, None, 2, 1), lambda: E.qk_norm_rotary_forward(x, x, 2, 2, Qn=x if bad is None else bad, Kn=line),
                     lambda: E.cross_attention_forward(x, bad, x, seqs, 2, 2, 1.0), lambda: E.cross_attention_backward(x, x, x, bad, x, lse, seqs, 2, 2, 1.0)):
            with pytest.raises(E.E2EGrecError):
                call()
    with pytest.raises(E.E2EGrecError):
        E.qk_norm_rotary_backward(line, None, line, None, 2, 1)
