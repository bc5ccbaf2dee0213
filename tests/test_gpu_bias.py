"""Attention with a bias by distance on the GPU against its 64-bit form."""
import math

import numpy as np
import pytest
import torch

import bias_oracle as F

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _randn(*shape, seed, dtype):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def _held(got, want, bound, what):
    got = got.double().cpu()
    hidden = torch.isinf(want)
    assert torch.equal(got[hidden], want[hidden]), what
    err = (got - want)[~hidden].abs()
    bad = ~(err <= bound[~hidden])
    assert not bad.any(), (what, int(bad.sum()), err.numel(), (err / bound[~hidden]).nan_to_num(nan=math.inf).max().item())


def _places(kind, ptr, rows, rng):
    """Positions of a packed matrix's rows: by row number, ascending times, unordered ones, ends of the range, all alike."""
    if kind == "rows":
        return None
    if kind == "alike":
        return torch.full((rows,), 12, dtype=torch.int32)
    if kind == "any":
        return torch.from_numpy(rng.integers(-300, 300, rows).astype(np.int32))
    if kind == "far":
        return torch.from_numpy(rng.choice(np.array([-2 ** 31, -2 ** 31 + 1, -5, 0, 7, 2 ** 31 - 1], dtype=np.int64), rows).astype(np.int32))
    pos = np.zeros(rows, dtype=np.int64)
    for s in range(len(ptr) - 1):
        pos[ptr[s]: ptr[s + 1]] = np.sort(rng.integers(0, 5000, ptr[s + 1] - ptr[s]))
    return torch.from_numpy(pos.astype(np.int32))


class Problem:
    """Ragged sequences with a gap before the first and rows behind the last; masked keys and rows outside hold NaN."""

    def __init__(self, q_lens, k_lens, heads, kv_heads, hd, dtype, edge, pos="times", masked=False, hides=(), seed=0, gap=3, spread=1.0, mean=0.0):
        rng = np.random.default_rng(seed)
        self.heads, self.kv_heads, self.hd, self.dtype, self.scale = heads, kv_heads, hd, dtype, hd ** -0.5
        self.q_ptr = torch.from_numpy(gap + np.concatenate([[0], np.cumsum(q_lens)])).long()
        self.k_ptr = torch.from_numpy(gap + np.concatenate([[0], np.cumsum(k_lens)])).long()
        nq, nk = int(self.q_ptr[-1]) + gap, int(self.k_ptr[-1]) + gap
        self.q, self.k = _randn(nq, heads * hd, seed=seed + 1, dtype=dtype) * spread, _randn(nk, kv_heads * hd, seed=seed + 2, dtype=dtype)
        self.v, self.g = (_randn(nk, kv_heads * hd, seed=seed + 3, dtype=dtype) + mean).to(dtype), _randn(nq, heads * hd, seed=seed + 4, dtype=dtype)
        self.edge = torch.tensor(edge, dtype=torch.int32)
        self.table = _randn(len(edge) + 1, heads, seed=seed + 5, dtype=F32) * 2
        for b, h, value in hides:
            self.table[b % (len(edge) + 1), h if h is None else h % heads] = value
        self.pos_q, self.pos_k = _places(pos, self.q_ptr.tolist(), nq, rng), _places(pos, self.k_ptr.tolist(), nk, rng)
        self.mask = None
        dead = torch.ones(nk, dtype=torch.bool)
        dead[int(self.k_ptr[0]): int(self.k_ptr[-1])] = False
        if masked:
            m = (rng.random(nk) > 0.3).astype(np.uint8)
            for s in range(1, len(k_lens), 4):                # every fourth sequence is hidden altogether
                m[int(self.k_ptr[s]): int(self.k_ptr[s + 1])] = 0
            self.mask = torch.from_numpy(m)
            dead |= self.mask == 0
        self.k_in, self.v_in, self.q_in, self.g_in = self.k.clone(), self.v.clone(), self.q.clone(), self.g.clone()
        self.k_in[dead], self.v_in[dead] = float("nan"), float("inf")
        for t in (self.q_in, self.g_in):
            t[: gap] = t[nq - gap:] = float("nan")
        self.live_q, self.live_k = slice(gap, nq - gap), slice(gap, nk - gap)

    def seqs(self, E, hints=True):
        mq = int((self.q_ptr[1:] - self.q_ptr[:-1]).max()) if hints is True else hints
        mk = int((self.k_ptr[1:] - self.k_ptr[:-1]).max()) if hints is True else hints
        return E.Sequences(self.q_ptr.cuda(), self.k_ptr.cuda(), mq, mk, None if self.mask is None else self.mask.cuda())

    def bias(self, E):
        c = lambda t: None if t is None else t.cuda()
        return E.RelativeBias(self.table.cuda(), self.edge.cuda(), c(self.pos_q), c(self.pos_k))

    def run(self, E, hints=True, wide=0, stream=None):
        def widen(t):         # `wide` more columns on either side: the distance of two rows need not be a multiple of a head
            side = torch.full((t.shape[0], wide), float("nan"), dtype=t.dtype)
            return torch.cat([side, t, side], 1).cuda()[:, wide: wide + t.shape[1]]
        q, k, v, g = (widen(t) for t in (self.q_in, self.k_in, self.v_in, self.g_in))
        fill = lambda t: widen(torch.full_like(t, 7.0))
        out, lse = fill(self.q), torch.full((self.q.shape[0], self.heads), 7.0).cuda()
        dq, dk, dv, dtable = fill(self.q), fill(self.k), fill(self.k), torch.full_like(self.table, 7.0).cuda()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        seqs, bias = self.seqs(E, hints), self.bias(E)
        torch.cuda.synchronize()
        E.biased_attention_forward(q, k, v, seqs, bias, self.heads, self.kv_heads, self.scale, out=out, lse=lse, status=status, stream=stream)
        E.biased_attention_backward(g, q, k, v, out, lse, seqs, bias, self.heads, self.kv_heads, self.scale, dQ=dq, dK=dk, dV=dv, dtable=dtable,
                                    status=status, stream=stream)
        torch.cuda.synchronize()
        assert int(status) == 0
        return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv, "dtable": dtable}

    def want(self):
        d = lambda t: t.double()
        return F.attention(d(self.q), d(self.k), d(self.v), self.q_ptr, self.k_ptr, self.heads, self.kv_heads, self.scale, self.edge, self.table,
                           self.pos_q, self.pos_k, self.mask, d(self.g), self.dtype, rounded_p=self.dtype == BF16)

    def check(self, res, want=None):
        want = want or self.want()
        for name, live in (("out", self.live_q), ("lse", self.live_q), ("dq", self.live_q), ("dk", self.live_k), ("dv", self.live_k)):
            got, (value, bound) = res[name], want[name]
            outside = torch.ones(got.shape[0], dtype=torch.bool)
            outside[live] = False
            assert (got.cpu()[outside] == 7.0).all(), name           # rows outside every sequence are left as they were
            _held(got[live], value[live], bound[live], name)
        _held(res["dtable"], *want["dtable"], "dtable")


def _go(*args, runs=(dict(),), **kw):
    import paper_2511_20564_b200 as E
    p = Problem(*args, **kw)
    want = p.want()
    for r in runs:
        p.check(p.run(E, **r), want)


LOG = F.edges(16, 2000)
BOTH = F.edges(32, 2000, True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,hd", [(1, 1, 8), (4, 4, 32), (6, 2, 40), (8, 1, 64), (4, 2, 128), (3, 3, 200), (2, 1, 256)])
def test_single_tokens(dtype, heads, kv_heads, hd):
    rng = np.random.default_rng(hd)
    k_lens = rng.integers(0, 130, 40)
    _go([1] * 40, k_lens, heads, kv_heads, hd, dtype, LOG, masked=heads > 3, runs=(dict(), dict(hints=0, wide=16)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 64), (6, 2, 36), (12, 1, 16)])
def test_stacks_of_tokens(dtype, heads, kv_heads, hd):
    hd = 40 if dtype == BF16 and hd == 36 else hd
    _go([3] * 50, [3] * 50, heads, kv_heads, hd, dtype, BOTH, pos="any", runs=(dict(), dict(hints=0)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 32), (6, 2, 40), (8, 1, 64), (2, 2, 128), (5, 5, 64), (10, 2, 96), (40, 1, 32), (2, 1, 256)])
@pytest.mark.parametrize("masked", [False, True])
def test_ragged_sequences(dtype, heads, kv_heads, hd, masked):
    _go([70, 0, 33, 129, 5, 260], [300, 45, 0, 140, 77, 513], heads, kv_heads, hd, dtype, BOTH, masked=masked,
        runs=(dict(), dict(hints=0), dict(wide=16)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pos", ["rows", "times", "any", "far", "alike"])
@pytest.mark.parametrize("edge", [[], [0], [-3, 2], list(range(-63, 64)), [-100, -100, -100, 0, 0, 50], [-(2 ** 31) + 1, 2 ** 31 - 1], F.edges(64, 1 << 30, True)])
def test_edges_and_positions(dtype, pos, edge):
    _go([1, 2, 40], [60, 7, 500], 4, 2, 64, dtype, edge, pos=pos)
    _go([200, 150], [300, 150], 4, 2, 64, dtype, edge, pos=pos, seed=1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [-math.inf, -1e30, torch.finfo(F32).min])
def test_buckets_that_hide(dtype, value):
    """Some buckets of some heads hidden, every bucket of one head: rows that see nothing get zeros."""
    hides = [(0, 0, value), (3, 1, value), (5, 2, value)] + [(b, 3, value) for b in range(16)]
    for lens in (([1] * 12, [50] * 12), ([130, 70, 300], [200, 64, 290]), ([3, 3], [4000, 9000])):
        _go(*lens, 4, 4, 64, dtype, LOG, hides=hides)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_long_histories(dtype):
    _go([1, 2, 1], [9000, 5000, 12_000], 8, 2, 64, dtype, F.edges(32, 5000), runs=(dict(), dict(hints=0)))
    _go([150, 3], [2500, 3000], 4, 2, 64, dtype, F.edges(32, 5000), masked=False, runs=(dict(), dict(hints=0)))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_values_with_much_in_common(dtype):
    """dP is nearly the same for all keys: what D lacks of it must not show in the table's gradient."""
    for lens in (([1] * 30, [100] * 30), ([200], [400]), ([2], [4000])):
        _go(*lens, 2, 2, 64, dtype, LOG, mean=4.0)


def test_repeats_bit_for_bit_and_streams():
    import paper_2511_20564_b200 as E
    for lens in (([1] * 60, [100] * 60), ([300, 200], [400, 350]), ([2], [4000])):
        for dtype in (BF16, F32):
            p = Problem(*lens, 4, 2, 64, dtype, BOTH)
            first = p.run(E)
            for stream in (None, torch.cuda.Stream(), None):
                for name, t in p.run(E, stream=stream).items():
                    assert torch.equal(t, first[name]), (name, lens)


def test_no_bias_is_the_attention_without():
    """A table of zeros: the same scores, so the same results up to what the order of sums leaves."""
    import paper_2511_20564_b200 as E
    for dtype in (BF16, F32):
        p = Problem([70, 1, 200], [300, 40, 260], 4, 2, 64, dtype, LOG)
        p.table.zero_()
        res = p.run(E)
        seqs = p.seqs(E)
        out, lse, _ = E.cross_attention_forward(p.q_in.cuda(), p.k_in.cuda(), p.v_in.cuda(), seqs, 4, 2, p.scale)
        tol = 2 ** -7 if dtype == BF16 else 1e-5
        assert (out[p.live_q].double() - res["out"][p.live_q].double()).abs().max() < tol and (lse[p.live_q] - res["lse"][p.live_q]).abs().max() < 1e-5


def test_empty_calls_zero_the_table_gradient():
    import paper_2511_20564_b200 as E
    for dtype in (BF16, F32):
        for q_lens, k_lens in (([0, 0], [5, 6]), ([4, 2], [0, 0]), ([], [])):
            p = Problem(q_lens, k_lens, 2, 2, 32, dtype, LOG, gap=0)
            res = p.run(E, hints=0)
            assert (res["dtable"] == 0).all() and (res["out"] == 0).all() and (res["dk"] == 0).all() and (res["dq"] == 0).all()
