"""Attention by distance, dropout, residual and layer norm in a row, as a block of a sequence model uses them: every stage against its 64-bit form
at the inputs it got, captured steps, graphs side by side, and the ways of the attention that only large tables or odd groups of heads take."""
import pytest
import torch

import bias_oracle as F
import residual_oracle as R
from test_gpu_bias import BOTH, Problem, _go
from test_gpu_residual import _held

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
LOG_NEAR = F.edges(16, 200, True)


def _same(got, want, problem):
    """Bit for bit, but for rows of no sequence, which nothing writes."""
    live = {"lse": problem.live_q, "dk": problem.live_k, "dv": problem.live_k}
    for n, t in got.items():
        rows = live.get(n, slice(None))
        assert torch.equal(t[rows], want[n][rows]), n


class Block:
    """y = norm(x + drop(attention(x, keys)));  out = y + drop(y).  The sequences are padded: rows of no sequence lie at both ends, finite."""

    def __init__(self, E, dtype, q_lens, k_lens, heads, kv_heads, hd, p=0.2, seed=0):
        self.E, self.dtype, self.p, self.seed = E, dtype, p, 77 + seed
        self.a = Problem(q_lens, k_lens, heads, kv_heads, hd, dtype, BOTH, masked=True, seed=seed)
        self.dim, rows = heads * hd, self.a.q.shape[0]
        gen = torch.Generator().manual_seed(seed + 50)
        self.gain, self.shift = 1 + 0.2 * torch.randn(self.dim, generator=gen), torch.randn(self.dim, generator=gen)
        self.dy = torch.randn(rows, self.dim, generator=gen).to(dtype)
        c = lambda t: t.cuda()
        self.x, self.k, self.v, self.g = c(self.a.q), c(self.a.k_in), c(self.a.v_in), c(self.dy)
        self.gains = c(self.gain), c(self.shift)
        self.seqs, self.bias = self.a.seqs(E), self.a.bias(E)
        self.step = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.out = torch.zeros_like(self.x)              # rows of no sequence are not written: zeros
        self.dq = torch.zeros_like(self.x)
        self.ws = [None, None, None]

    def plans(self):
        return [self.E.Dropout(self.p, self.seed, place=i, step_dev=self.step) for i in (0, 1)]

    def run(self):
        E, a, plans = self.E, self.a, self.plans()
        att, lse, self.ws[0] = E.biased_attention_forward(self.x, self.k, self.v, self.seqs, self.bias, a.heads, a.kv_heads, a.scale, out=self.out,
                                                          status=self.status, ws=self.ws[0])
        y, z, stats = E.layer_norm_forward(att, *self.gains, residual=self.x, drop=plans[0], keep_sum=True)
        out = E.dropout(y, plans[1], residual=y)
        # backward
        dy = E.dropout(self.g, plans[1], residual=self.g)
        datt, dx, dgain, dshift, self.ws[1] = E.layer_norm_backward(dy, att, stats, self.gains[0], residual=self.x, drop=plans[0], ws=self.ws[1])
        dq, dk, dv, dtable, self.ws[2] = E.biased_attention_backward(datt, self.x, self.k, self.v, att, lse, self.seqs, self.bias, a.heads, a.kv_heads,
                                                                     a.scale, dQ=self.dq, status=self.status, ws=self.ws[2])
        return dict(att=att, lse=lse, y=y, z=z, out=out, dy=dy, datt=datt, dx=dx, dgain=dgain, dshift=dshift, dq=dq, dk=dk, dv=dv, dtable=dtable)

    def check(self, res, step=0):
        a, d = self.a, lambda t: t.double().cpu()
        f = [R.factors(*self.x.shape, self.p, self.seed, i, step) for i in (0, 1)]
        assert int(self.status) == 0
        want = F.attention(d(a.q), d(a.k), d(a.v), a.q_ptr, a.k_ptr, a.heads, a.kv_heads, a.scale, a.edge, a.table, a.pos_q, a.pos_k, a.mask,
                           d(res["datt"]), self.dtype, rounded_p=self.dtype == BF16)
        for name, got, live in (("out", "att", a.live_q), ("lse", "lse", a.live_q), ("dq", "dq", a.live_q), ("dk", "dk", a.live_k), ("dv", "dv", a.live_k)):
            _held_where_finite(res[got][live], want[name][0][live], want[name][1][live], name)
        _held(res["dtable"], *want["dtable"], "dtable")
        assert (res["dq"][: a.live_q.start] == 0).all() and (res["att"][a.live_q.stop:] == 0).all()
        norm = R.norm(d(res["att"]), d(self.x), f[0], self.gain, self.shift, 1e-5, self.dtype, d(res["dy"]))
        for name, got in (("y", "y"), ("z", "z"), ("dx", "datt"), ("dr", "dx"), ("dgain", "dgain"), ("dshift", "dshift")):
            _held(res[got], *norm[name], name)
        h = R.HALF[self.dtype]
        for src, got in ((res["y"], "out"), (self.g, "dy")):
            z, bz = R.total(d(src), d(src), f[1])
            _held(res[got], z, h * z.abs() + (1 + h) * bz, got)


def _held_where_finite(got, want, bound, what):
    fin = torch.isfinite(want)
    assert torch.equal(got.double().cpu()[~fin], want[~fin]), what
    _held(got.cpu()[fin], want[fin], bound[fin], what)


SHAPES = [([1] * 40, [30] * 40, 4, 4, 32), ([70, 1, 0, 200], [90, 300, 20, 260], 4, 2, 64), ([2, 1], [3000, 2500], 8, 2, 16)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_block_forward_and_backward(dtype, shape):
    import paper_2511_20564_b200 as E
    b = Block(E, dtype, *shape)
    b.check(b.run())


def _capture(b):
    b.run()                                              # workspaces as a program has them: made before, kept
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = b.run()
    return graph, res


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_captured_block_repeats_the_eager_one(dtype, shape):
    import paper_2511_20564_b200 as E
    b = Block(E, dtype, *shape)
    graph, res = _capture(b)
    for k in (3, 0, 3):
        b.step.fill_(k)
        b.status.zero_()
        for t in res.values():
            if t is not res["att"] and t is not res["dq"]:
                t.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        b.check(res, k)
        got = {n: t.clone() for n, t in res.items()}
        _same(b.run(), got, b.a)


def test_graphs_side_by_side_and_one_after_another():
    """Two captured blocks with their own workspaces at once on two streams; then both with one workspace, in turn on one stream."""
    import paper_2511_20564_b200 as E
    blocks = [Block(E, BF16, [150, 70], [300, 200], 4, 2, 64, seed=i * 100) for i in (0, 1)]
    made = [_capture(b) for b in blocks]
    first = []
    for g, res in made:
        g.replay()
        torch.cuda.synchronize()
        first.append({n: t.clone() for n, t in res.items()})
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(20):
        for s, (g, _r) in zip(streams, made):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for b, f, (_g, res) in zip(blocks, first, made):
        _same(res, f, b.a)
    blocks[1].ws = blocks[0].ws
    graph, res = _capture(blocks[1])
    for _ in range(3):
        made[0][0].replay()
        graph.replay()
    made[0][0].replay()
    torch.cuda.synchronize()
    _same(made[0][1], first[0], blocks[0].a)
    _same(res, first[1], blocks[1].a)
    for b in blocks:
        assert int(b.status) == 0


def test_calls_at_once_on_two_streams():
    import paper_2511_20564_b200 as E
    for lens in (([1] * 60, [100] * 60), ([300, 200], [400, 350]), ([2], [4000])):
        for dtype in (BF16, F32):
            ps = [Problem(*lens, 4, 2, 64, dtype, BOTH, seed=i) for i in (0, 9)]
            first = [p.run(E) for p in ps]
            args = [(p.q_in.cuda(), p.k_in.cuda(), p.v_in.cuda(), p.seqs(E), p.bias(E), p.g_in.cuda()) for p in ps]
            streams = [torch.cuda.Stream() for _ in ps]
            torch.cuda.synchronize()
            got = []
            for _ in range(3):
                for s, p, f, (q, k, v, seqs, bias, g) in zip(streams, ps, first, args):
                    with torch.cuda.stream(s):
                        got.append((f, E.biased_attention_backward(g, q, k, v, f["out"], f["lse"], seqs, bias, 4, 2, p.scale)))
            torch.cuda.synchronize()
            for i, (f, (dq, dk, dv, dtable, _)) in enumerate(got):
                live_q, live_k = ps[i % 2].live_q, ps[i % 2].live_k
                assert torch.equal(dtable, f["dtable"]) and torch.equal(dq[live_q], f["dq"][live_q])
                assert torch.equal(dk[live_k], f["dk"][live_k]) and torch.equal(dv[live_k], f["dv"][live_k])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,buckets", [(128, 128, 64), (64, 4, 128), (32, 1, 100), (20, 4, 64), (24, 2, 128), (512, 512, 128), (1, 1, 1), (96, 96, 3), (10, 1, 128),
                                                    (8, 1, 56), (4, 1, 110), (9, 1, 64), (8, 2, 128), (3, 1, 128)])
def test_large_tables_and_odd_groups(dtype, heads, kv_heads, buckets):
    """Tables that no block's shared memory holds whole, bins that it does not hold, groups of heads that divide no tile."""
    hd = 8 if heads > 64 else 16
    edge = [4 * (i - buckets // 2) for i in range(buckets - 1)]
    for lens, pos in ((([1, 2, 1], [60, 7, 90]), "any"), (([40, 90], [150, 33]), "any"), (([2], [2500]), "times")):
        _go(*lens, heads, kv_heads, hd, dtype, edge, pos=pos)


@pytest.mark.parametrize("heads,kv_heads,buckets", [(10, 1, 128), (8, 1, 56), (4, 4, 127), (4, 2, 128)])
def test_large_tables_beside_wide_heads(heads, kv_heads, buckets):
    """Values with much in common: what the stored out lacks must not show in the table's gradient, whichever kernel forms it."""
    edge = [9 * (i - buckets // 2) for i in range(buckets - 1)]
    for dtype in (BF16, F32):
        _go([150, 0, 33], [333, 40, 128], heads, kv_heads, 128, dtype, edge, pos="times", mean=4.0, runs=(dict(), dict(hints=0)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd", [128, 100, 72, 64, 32])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (2, 1), (3, 3)])
def test_every_size_of_table_beside_the_tiles(dtype, hd, heads, kv_heads):
    """What a bias takes beside the tiles grows by little steps: none of them may tip over what a block is given."""
    hd = (hd + 7) // 8 * 8
    for buckets in [1, 2, 4, 6, 7, 8, 9, 10, 11, 12, 14, 16, 20, 24, 32, 47, 63, 80, 101, 128]:
        _go([70], [130], heads, kv_heads, hd, dtype, [3 * (i - buckets // 2) for i in range(buckets - 1)], pos="rows")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 32), (6, 2, 72), (2, 1, 256), (3, 3, 128)])
def test_sequences_longer_than_their_hints(dtype, heads, kv_heads, hd):
    """Hints choose kernels, longer sequences are still right."""
    for lens in (([1, 5, 0, 2], [40, 300, 7, 90]), ([70, 3, 130], [300, 1000, 150]), ([1, 1], [3000, 10])):
        _go(*lens, heads, kv_heads, hd, dtype, BOTH, masked=True, mean=1.0, runs=(dict(hints=1), dict(hints=3), dict(hints=33), dict(hints=5000)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("q_len", [1, 40, 200])
def test_offsets_out_of_order_are_reported_and_stay_in_bounds(q_len, dtype):
    import paper_2511_20564_b200 as E
    x = torch.randn(3 * q_len, 64, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    pos = torch.arange(3 * q_len, dtype=torch.int32, device="cuda")
    bias = E.RelativeBias(torch.ones(32, 2, device="cuda"), E.relative_edges(32, 1000), pos, pos)
    good = torch.tensor([0, q_len, 2 * q_len, 3 * q_len], device="cuda")
    for bad in ([0, 10 ** 12, 2 * q_len, 3 * q_len], [-5, q_len, 2 * q_len, 3 * q_len], [0, 2 * q_len, q_len, 3 * q_len]):
        bad = torch.tensor(bad, device="cuda")
        for hint in (q_len, 0):
            for seqs in (E.Sequences(bad, good, hint, hint), E.Sequences(good, bad, hint, hint)):
                status = torch.zeros(1, dtype=torch.int32, device="cuda")
                out, lse, _ = E.biased_attention_forward(x, x, x, seqs, bias, 2, 2, 0.125, status=status)
                assert status.item() == 1
                status.zero_()
                E.biased_attention_backward(x, x, x, x, torch.zeros_like(x), torch.zeros_like(lse), seqs, bias, 2, 2, 0.125, status=status)
                assert status.item() == 1
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_table_without_a_gradient(dtype):
    """table_grad=False: nothing of the table's gradient is formed, the others are within the same bounds."""
    import paper_2511_20564_b200 as E
    for lens in (([1] * 30, [100] * 30), ([70, 3, 200], [300, 40, 700]), ([2, 1], [4000, 100])):
        p = Problem(*lens, 4, 2, 64, dtype, BOTH, masked=True)
        res, want = p.run(E), p.want()
        args = [t.cuda() for t in (p.g_in, p.q_in, p.k_in, p.v_in)]
        dq, dk, dv, dtable, _ = E.biased_attention_backward(*args, res["out"], res["lse"], p.seqs(E), p.bias(E), 4, 2, p.scale, table_grad=False)
        assert dtable is None
        for got, name, live in ((dq, "dq", p.live_q), (dk, "dk", p.live_k), (dv, "dv", p.live_k)):
            _held(got[live], want[name][0][live], want[name][1][live], name)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_further_apart_than_32_bits(dtype):
    """One matrix of rows 2^26 elements apart holds everything: its last rows lie beyond 2^31 elements."""
    import paper_2511_20564_b200 as E
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    for lens in (([45], [45]), ([1] * 45, [1] * 45)):
        p = Problem(*lens, 4, 2, 32, dtype, LOG_NEAR, gap=0, pos="any")
        want, rows = p.want(), 45
        big = torch.empty(rows, 1 << 26, dtype=dtype, device="cuda")
        place = lambda i, t: big[:, i * 256: i * 256 + t.shape[1]].copy_(t)
        q, k, v, g = (place(i, t) for i, t in enumerate((p.q, p.k, p.v, p.g)))
        out, dq, dk, dv, y, dx = (big[:, (4 + i) * 256: (4 + i) * 256 + t.shape[1]] for i, t in enumerate((p.q, p.q, p.k, p.k, p.q, p.q)))
        seqs, bias = p.seqs(E), p.bias(E)
        _, lse, _ = E.biased_attention_forward(q, k, v, seqs, bias, 4, 2, p.scale, out=out)
        dtable = E.biased_attention_backward(g, q, k, v, out, lse, seqs, bias, 4, 2, p.scale, dQ=dq, dK=dk, dV=dv)[3]
        for name, t in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv), ("dtable", dtable)):
            _held(t, *want[name], name)
        plan = E.Dropout(0.3, 5)
        f, d = R.factors(rows, 128, 0.3, 5), lambda t: t.double().cpu()
        norm = R.norm(d(out), d(q), f, None, None, 1e-5, dtype, d(g))
        _, _, stats = E.layer_norm_forward(out, residual=q, drop=plan, Y=y)
        dgain = E.layer_norm_backward(g, out, stats, residual=q, drop=plan, dX=dx)[2]
        for name, t in (("y", y), ("dx", dx), ("dgain", dgain)):
            _held(t, *norm[name], name)
        E.dropout(q, plan, residual=g, out=y)
        z, bz = R.total(d(q), d(g), f)
        _held(y, z, R.HALF[dtype] * z.abs() + (1 + R.HALF[dtype]) * bz, "dropout")
        del big, q, k, v, g, out, dq, dk, dv, y, dx
