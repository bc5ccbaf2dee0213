"""Attention of ragged sequences of tokens to ragged sequences of states, against its 64-bit form."""
import math

import numpy as np
import pytest
import torch

import fusion_oracle as F

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
    assert not bad.any(), (what, int(bad.sum()), (err / bound[~hidden]).max().item())


class Problem:
    """Ragged sequences with a gap before the first and rows behind the last; masked keys and rows outside hold NaN."""

    def __init__(self, q_lens, k_lens, heads, kv_heads, hd, dtype, masked=False, seed=0, gap=3, scale=None, spread=1.0):
        self.heads, self.kv_heads, self.hd, self.dtype = heads, kv_heads, hd, dtype
        self.scale = hd ** -0.5 if scale is None else scale
        self.q_ptr = torch.from_numpy(gap + np.concatenate([[0], np.cumsum(q_lens)])).long()
        self.k_ptr = torch.from_numpy(gap + np.concatenate([[0], np.cumsum(k_lens)])).long()
        nq, nk = int(self.q_ptr[-1]) + gap, int(self.k_ptr[-1]) + gap
        self.q, self.k = _randn(nq, heads * hd, seed=seed + 1, dtype=dtype) * spread, _randn(nk, kv_heads * hd, seed=seed + 2, dtype=dtype)
        self.v, self.g = _randn(nk, kv_heads * hd, seed=seed + 3, dtype=dtype), _randn(nq, heads * hd, seed=seed + 4, dtype=dtype)
        self.mask = None
        if masked:
            rng = np.random.default_rng(seed)
            m = (rng.random(nk) > 0.3).astype(np.uint8)
            for s in range(0, len(k_lens), 4):                # every fourth sequence is hidden altogether
                m[int(self.k_ptr[s + 1]) - k_lens[s]: int(self.k_ptr[s + 1])] = 0 if s else m[int(self.k_ptr[0]): int(self.k_ptr[1])]
            self.mask = torch.from_numpy(m)
        dead = torch.ones(nk, dtype=torch.bool)
        dead[int(self.k_ptr[0]): int(self.k_ptr[-1])] = False
        if masked:
            dead |= self.mask == 0
        self.k_in, self.v_in = self.k.clone(), self.v.clone()
        self.k_in[dead], self.v_in[dead] = float("nan"), float("inf")
        self.q_in, self.g_in = self.q.clone(), self.g.clone()
        for t in (self.q_in, self.g_in):
            t[: gap] = t[nq - gap:] = float("nan")
        self.live_q, self.live_k = slice(gap, nq - gap), slice(gap, nk - gap)

    def seqs(self, E, hints=True):
        mq = int((self.q_ptr[1:] - self.q_ptr[:-1]).max()) if hints is True else hints
        mk = int((self.k_ptr[1:] - self.k_ptr[:-1]).max()) if hints is True else hints
        return E.Sequences(self.q_ptr.cuda(), self.k_ptr.cuda(), mq, mk, None if self.mask is None else self.mask.cuda())

    def run(self, E, hints=True, backward=True, wide=0):
        cu = lambda t: t.cuda()
        if wide:          # column ranges of wider matrices, and results into such ranges
            def widen(t):         # `wide` more columns on either side: the distance of two rows need not be a multiple of a head
                side = torch.full((t.shape[0], wide), float("nan"), dtype=t.dtype)
                return torch.cat([side, t, side], 1).cuda()[:, wide: wide + t.shape[1]]
        else:
            widen = cu
        q, k, v, g = widen(self.q_in), widen(self.k_in), widen(self.v_in), widen(self.g_in)
        fill = lambda t: widen(torch.full_like(t, 7.0))
        out, lse = fill(self.q), torch.full((self.q.shape[0], self.heads), 7.0).cuda()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        seqs = self.seqs(E, hints)
        E.cross_attention_forward(q, k, v, seqs, self.heads, self.kv_heads, self.scale, out=out, lse=lse, status=status)
        res = {"out": out, "lse": lse}
        if backward:
            # what rows outside the sequences hold has no influence either
            o = out.clone()
            o[: self.live_q.start] = float("nan")
            dq, dk, dv, _ = E.cross_attention_backward(g, q, k, v, o, lse, seqs, self.heads, self.kv_heads, self.scale, dQ=fill(self.q),
                                                       dK=fill(self.k), dV=fill(self.v), status=status)
            res.update(dq=dq, dk=dk, dv=dv)
        assert status.item() == 0
        return res

    def want(self, backward=True, rounded_p=None):
        rounded = self.dtype == BF16 if rounded_p is None else rounded_p
        d = lambda t: t.double()
        return F.attention(d(self.q), d(self.k), d(self.v), self.q_ptr, self.k_ptr, self.heads, self.kv_heads, self.scale, self.mask,
                           d(self.g) if backward else None, self.dtype, rounded)

    def check(self, got, want):
        for name, (val, bound) in want.items():
            rows = self.live_k if name in ("dk", "dv") else self.live_q
            assert (got[name][: rows.start] == 7).all() and (got[name][rows.stop:] == 7).all(), name     # left as they were
            _held(got[name][rows], val[rows], bound[rows], name)


LENGTHS = {
    "ones": ([1] * 9, [1] * 9),
    "single tokens": ([1, 1, 0, 1, 1, 1, 1], [100, 0, 17, 64, 65, 1, 200]),
    "a few tokens": ([3, 2, 0, 3, 1, 4], [3, 40, 9, 129, 0, 64]),
    "ragged": ([37, 1, 0, 130, 64], [77, 211, 5, 128, 0]),
    "tiles": ([128, 129, 127, 256], [128, 127, 129, 256]),
    "long keys": ([2, 1, 1], [5003, 1, 2048]),
    "long both": ([300, 515], [700, 333]),
}
HEADS = [(4, 4, 32), (2, 1, 64), (3, 3, 128), (6, 2, 40), (8, 2, 96), (2, 2, 16), (1, 1, 256), (16, 1, 8), (5, 5, 80)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("masked", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("heads,kv_heads,hd", HEADS)
@pytest.mark.parametrize("lengths", LENGTHS)
def test_forward_and_backward(lengths, heads, kv_heads, hd, masked, dtype):
    import paper_2511_20564_b200 as E
    p = Problem(*LENGTHS[lengths], heads, kv_heads, hd, dtype, masked)
    p.check(p.run(E), p.want())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lengths", ["single tokens", "ragged"])
def test_column_ranges_hints_and_repetition(lengths, dtype):
    """Matrices that are column ranges of wider ones; hints that are missing or far too small; the same bits every time."""
    import paper_2511_20564_b200 as E
    p = Problem(*LENGTHS[lengths], 4, 2, 64, dtype, True)
    want = p.want()
    first = p.run(E)
    p.check(first, want)
    again = p.run(E)
    for name in first:
        assert torch.equal(first[name], again[name]), name
    p.check(p.run(E, wide=8), want)
    p.check(p.run(E, wide=128), want)
    p.check(p.run(E, hints=0), want)
    p.check(p.run(E, hints=1), want)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lengths", ["single tokens", "ragged", "long keys"])
def test_sharp_and_rising_scores(lengths, dtype):
    """Scores of a hundred and more, rising along the keys, so that the running maximum moves all the time."""
    import paper_2511_20564_b200 as E
    p = Problem(*LENGTHS[lengths], 2, 2, 64, dtype, scale=1.0, spread=2.0)
    ramp = torch.linspace(0.2, 2.0, p.k.shape[0])[:, None].to(dtype)
    p.k, p.k_in = (p.k.abs() * ramp).to(dtype), (p.k_in.abs() * ramp).to(dtype)
    p.q, p.q_in = p.q.abs(), p.q_in.abs()
    p.check(p.run(E), p.want())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,hd", [(130, 1, 8), (21, 3, 16), (48, 2, 128)])
def test_many_query_heads_per_key_head(heads, kv_heads, hd, dtype):
    """Groups larger than a tile has rows, and groups that do not divide its rows."""
    import paper_2511_20564_b200 as E
    p = Problem([3, 1, 0, 20], [70, 200, 9, 131], heads, kv_heads, hd, dtype, True)
    p.check(p.run(E), p.want())


def test_two_threads_at_once():
    """Calls from two host threads on streams of their own, kernels of every kind used for the first time by both."""
    import threading
    import paper_2511_20564_b200 as E
    problems = [Problem([3, 1, 40], [50, 260, 140], 4, 2, hd, dtype, seed=i, gap=0) for i, (hd, dtype) in enumerate([(48, BF16), (24, F32), (8, BF16), (112, F32)])]
    results, errors = {}, []

    def work(side):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(3):
                    for i, p in enumerate(problems):
                        results[side, i] = p.run(E)
                torch.cuda.current_stream().synchronize()
        except Exception as e:          # handed to the test's own thread
            errors.append(e)

    threads = [threading.Thread(target=work, args=(side,)) for side in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for i, p in enumerate(problems):
        p.check(results[0, i], p.want())
        for name, value in results[0, i].items():
            assert torch.equal(value, results[1, i][name])


def test_no_sequences_no_rows_no_lse():
    import paper_2511_20564_b200 as E
    x = _randn(4, 64, seed=1, dtype=BF16).cuda()
    ptr = torch.zeros(1, dtype=torch.int64, device="cuda")
    out = torch.full_like(x, 7.0)
    E.cross_attention_forward(x, x, x, E.Sequences(ptr, ptr), 2, 2, 1.0, out=out)
    assert (out == 7).all()
    two = torch.tensor([0, 2, 4], device="cuda")
    none = x[:0]
    E.cross_attention_forward(none, x, x, E.Sequences(torch.zeros(3, dtype=torch.int64, device="cuda"), two), 2, 2, 1.0)
    out, lse, _ = E.cross_attention_forward(x, none, none, E.Sequences(two, torch.zeros(3, dtype=torch.int64, device="cuda")), 2, 2, 1.0)
    assert not out.any() and (lse == -math.inf).all()
    dq, dk, dv, _ = E.cross_attention_backward(x, x, none, none, out, lse, E.Sequences(two, torch.zeros(3, dtype=torch.int64, device="cuda")), 2, 2, 1.0)
    assert not dq.any() and dk.shape == (0, 64)
    dq, dk, dv, _ = E.cross_attention_backward(none, none, x, x, none, lse[:0], E.Sequences(torch.zeros(3, dtype=torch.int64, device="cuda"), two), 2, 2, 1.0)
    assert not dk.any() and not dv.any()
    a, no, _ = E.cross_attention_forward(x, x, x, E.Sequences(two, two), 2, 2, 1.0, keep_lse=False)
    b, _, _ = E.cross_attention_forward(x, x, x, E.Sequences(two, two), 2, 2, 1.0)
    assert no is None and torch.equal(a, b)


@pytest.mark.parametrize("q_len", [1, 40])
def test_offsets_out_of_order_are_reported_and_stay_in_bounds(q_len):
    import paper_2511_20564_b200 as E
    x = _randn(3 * q_len, 64, seed=1, dtype=BF16).cuda()
    good = torch.tensor([0, q_len, 2 * q_len, 3 * q_len], device="cuda")
    for bad in ([0, 10 ** 12, 2 * q_len, 3 * q_len], [-5, q_len, 2 * q_len, 3 * q_len], [0, 2 * q_len, q_len, 3 * q_len]):
        bad = torch.tensor(bad, device="cuda")
        for seqs in (E.Sequences(bad, good, q_len, q_len), E.Sequences(good, bad, q_len, q_len)):
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            out, lse, _ = E.cross_attention_forward(x, x, x, seqs, 2, 2, 0.125, status=status)
            assert status.item() == 1
            E.cross_attention_backward(x, x, x, x, torch.zeros_like(x), torch.zeros_like(lse), seqs, 2, 2, 0.125, status=status)
            assert status.item() == 1
    torch.cuda.synchronize()


def test_other_streams_and_graphs():
    """A call on another stream than the current one; forward and backward captured together and replayed on new values, beside
    eager calls that have workspaces of their own."""
    import paper_2511_20564_b200 as E
    p = Problem([1, 3, 70], [50, 260, 140], 4, 2, 64, BF16, gap=0)
    q, k, v, g = (t.cuda() for t in (p.q, p.k, p.v, p.g))
    seqs = p.seqs(E)

    def both(stream=None):
        out, lse, w = E.cross_attention_forward(q, k, v, seqs, 4, 2, p.scale, stream=stream)
        return [out, lse] + list(E.cross_attention_backward(g, q, k, v, out, lse, seqs, 4, 2, p.scale, stream=stream)[:3]), w

    want, _ = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _ = both(side)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept, w = both()
    q2 = _randn(*p.q.shape, seed=50, dtype=BF16).cuda()
    q.copy_(q2)
    want, _ = both()
    graph.replay()
    again, _ = both()
    torch.cuda.synchronize()
    for a, b, c in zip(want, kept, again):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("q_len", [1, 200])
def test_rows_beyond_two_gigabytes(q_len):
    """Keys and values whose rows lie 64 MB apart: offsets pass 32 bits in elements and in bytes."""
    import paper_2511_20564_b200 as E
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("not enough memory")
    n, hd, ld = 200, 64, 1 << 25
    base = torch.empty(n * ld, dtype=BF16, device="cuda")
    k, v = base.as_strided((n, 2 * hd), (ld, 1)), base.as_strided((n, 2 * hd), (ld, 1), 4096)
    small = [_randn(n, 2 * hd, seed=s, dtype=BF16).cuda() for s in (1, 2)]
    k.copy_(small[0])
    v.copy_(small[1])
    q = _randn(q_len, 4 * hd, seed=3, dtype=BF16).cuda()
    ptr = lambda m: torch.tensor([0, m], device="cuda")
    seqs = E.Sequences(ptr(q_len), ptr(n), q_len, n)
    a, la, _ = E.cross_attention_forward(q, k, v, seqs, 4, 2, 0.125)
    b, lb, _ = E.cross_attention_forward(q, *small, seqs, 4, 2, 0.125)
    assert torch.equal(a, b) and torch.equal(la, lb)
    dk, dv = base.as_strided((n, 2 * hd), (ld, 1), 8192), base.as_strided((n, 2 * hd), (ld, 1), 12288)
    ga = E.cross_attention_backward(q, q, k, v, a, la, seqs, 4, 2, 0.125, dK=dk, dV=dv)
    gb = E.cross_attention_backward(q, q, *small, b, lb, seqs, 4, 2, 0.125)
    for x, y in zip(ga[:3], gb[:3]):
        assert torch.equal(x, y)


@pytest.mark.parametrize("n_seq,heads,kv_heads,hd,dtype", [(24, 4, 2, 32, BF16), (24, 4, 4, 16, F32), (70, 2, 2, 64, BF16)])
def test_encoder_states_through_norm_rotation_attention_and_back(n_seq, heads, kv_heads, hd, dtype):
    """The operators as they are used: the encoder's embeddings of a batch are the states of ragged sequences; queries and keys
    are normalised and rotated, tokens attend, and the gradient goes back through all of it to the encoder's weights and rows."""
    import oracle
    import paper_2511_20564_b200 as E
    import synth_inputs as S
    w = S.WORKLOADS["tiny"]
    d = kv_heads * hd
    indptr, indices, _ = S.build_graph(w)
    n_states = w.batch
    seeds = S.seed_batch(w.n_nodes, n_states, w.seed, 0)
    X_h = S.normal_features(w.n_nodes, w.dim, 3)
    Ws_h = [S.glorot_uniform(w.hidden, 2 * w.dim, 5, 50), S.glorot_uniform(d, 2 * w.hidden, 5, 51)]
    if dtype == BF16:
        X_h, Ws_h = S.to_bf16_values(X_h), [S.to_bf16_values(W) for W in Ws_h]
    cu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    X, Ws = cu(X_h).to(dtype), [cu(W).to(dtype) for W in Ws_h]
    blocks = E.Blocks(w.n_nodes, n_states, w.fanouts)
    E.sample_khop(cu(indptr), cu(indices), cu(seeds), blocks, w.seed, 0)
    H, ctx = E.sage_forward(blocks, X, Ws, acts=[0, 0])
    H = H[:n_states]
    rng = np.random.default_rng(n_seq)
    cuts = np.sort(rng.integers(0, n_states + 1, n_seq - 1))
    k_ptr = np.concatenate([[0], cuts, [n_states]])
    q_ptr = np.concatenate([[0], np.cumsum(rng.integers(0, 4, n_seq))])
    nq = int(q_ptr[-1])
    q, g = _randn(nq, heads * hd, seed=1, dtype=dtype), _randn(nq, heads * hd, seed=2, dtype=dtype)
    wq, wk = 1 + 0.1 * _randn(hd, seed=3, dtype=F32), 1 + 0.1 * _randn(hd, seed=4, dtype=F32)
    pos = lambda ptr: torch.cat([torch.arange(int(b - a)) for a, b in zip(ptr[:-1], ptr[1:])]).to(torch.int32)
    pq, pk = pos(q_ptr), pos(k_ptr)
    f = E.rotary_frequencies(hd)
    plan = dict(freqs=f, pos_q=pq.cuda(), pos_k=pk.cuda())
    seqs = E.Sequences(cu(q_ptr), cu(k_ptr), 3, n_states)
    qd, gd, wqd, wkd = q.cuda(), g.cuda(), wq.cuda(), wk.cuda()
    qn, kn = E.qk_norm_rotary_forward(qd, H, heads, kv_heads, wqd, wkd, **plan)
    out, lse, _ = E.cross_attention_forward(qn, kn, H, seqs, heads, kv_heads, hd ** -0.5)
    dqn, dkn, dv, _ = E.cross_attention_backward(gd, qn, kn, H, out, lse, seqs, heads, kv_heads, hd ** -0.5)
    dq, dk, dwq, dwk, _ = E.qk_norm_rotary_backward(dqn, dkn, qd, H, heads, kv_heads, wqd, wkd, **plan)
    dH = torch.zeros(blocks.caps[0][0], d, dtype=dtype, device="cuda")
    dH[:n_states] = (dk.float() + dv.float()).to(dtype)
    dWs, dX = E.sage_backward(blocks, X, Ws, ctx, dH, acts=[0, 0])
    torch.cuda.synchronize()
    # the same in 64 bits from the encoder's stored embeddings
    c = lambda t: t.double().cpu()
    fr = F.frequencies(hd)
    wqn = F.rotate(F.norm(c(q), heads, c(wq), 1e-6), heads, fr, pq)
    wkn = F.rotate(F.norm(c(H), kv_heads, c(wk), 1e-6), kv_heads, fr, pk)
    res = F.attention(wqn, wkn, c(H), q_ptr, k_ptr, heads, kv_heads, hd ** -0.5, None, c(g), dtype)
    wdq, wdwq, _, _ = F.norm_rotary_backward(res["dq"][0], c(q), heads, c(wq), 1e-6, fr, pq)
    wdk, wdwk, _, _ = F.norm_rotary_backward(res["dk"][0], c(H), kv_heads, c(wk), 1e-6, fr, pk)
    wdH = wdk + res["dv"][0]
    # A chain of storages: in 16 bits every stored matrix is off by 2^-8 of its values at most, and what follows passes that on
    # through sums of some tens of terms; relative to the root mean square of the result that stays below twelve such steps.
    tol = 12 * F.HALF[dtype] if dtype == BF16 else 2.0 ** -15
    for name, got, want in (("out", out, res["out"][0]), ("dq", dq, wdq), ("dwq", dwq, wdwq), ("dwk", dwk, wdwk), ("dH", dH[:n_states], wdH)):
        err = (c(got) - want).norm() / want.norm()
        assert err <= tol, (name, err.item())
    # ... and the encoder's backward pass takes it on as it takes any gradient (linear encoder: no sign to decide; a handful of
    # storages of at most half a step each, or fp32 sums of some hundred terms)
    blocks_o = oracle.sample_khop(indptr, indices, seeds, w.fanouts, w.seed, 0)
    H_o, ctx_o = oracle.sage_forward(blocks_o, X_h, Ws_h, acts=[0, 0], bf16=dtype == BF16)
    dW_o, _, dX_o = oracle.sage_backward(blocks_o, ctx_o, Ws_h, dH[:n_states].float().cpu().numpy(), acts=[0, 0], bf16=dtype == BF16)
    n_src = blocks_o[-1]["n_src"]
    for got, want in [(dX[:n_src], dX_o)] + list(zip(dWs, dW_o)):
        want = torch.from_numpy(np.asarray(want, np.float64))
        assert (c(got) - want).norm() / want.norm() <= (2e-2 if dtype == BF16 else 1e-4)
