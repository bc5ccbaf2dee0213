"""Dropout and layer norm on the GPU against their 64-bit forms."""
import pytest
import torch

import residual_oracle as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _randn(*shape, seed, dtype, mean=0.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) + mean).to(dtype)


def _held(got, want, bound, what):
    err = (got.double().cpu() - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), (err / bound).nan_to_num().max().item())


def _wide(t, side):
    """The same matrix as a column range of a wider one, whose other columns hold NaN."""
    s = torch.full((t.shape[0], side), float("nan"), dtype=t.dtype)
    return torch.cat([s, t, s], 1).cuda()[:, side: side + t.shape[1]]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,dim", [(0, 64), (1, 8), (1, 16), (7, 40), (33, 256), (1000, 72), (4099, 516), (70_001, 8), (3, 8192)])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(dtype, rows, dim, residual):
    import paper_2511_20564_b200 as E
    dim = dim // 8 * 8 if dtype == BF16 else dim
    x, r = _randn(rows, dim, seed=1, dtype=dtype), _randn(rows, dim, seed=2, dtype=dtype) if residual else None
    for p, seed, place, step in ((0.0, 5, 0, 0), (0.3, 0x1234_5678_9ABC_DEF0, 7, 0xFFFF_FFFF), (0.999_999, 5, (1 << 31) - 1, 3)):
        f = R.factors(rows, dim, p, seed, place, step)
        z, bz = R.total(x.double(), None if r is None else r.double(), f)
        plan = E.Dropout(p, seed, place=place, step=step)
        side = 16 // x.element_size()
        outs = [E.dropout(x.cuda(), plan, residual=None if r is None else r.cuda()),
                E.dropout(_wide(x, side), plan, residual=None if r is None else _wide(r, side), out=_wide(torch.full_like(x, 7), side))]
        inplace = x.cuda()
        E.dropout(inplace, plan, residual=None if r is None else r.cuda(), out=inplace)
        for y in outs + [inplace]:
            _held(y, z, R.HALF[dtype] * z.abs() + (1 + R.HALF[dtype]) * bz, (p, residual))
            if r is None:
                assert torch.equal(y.cpu() == 0, (f == 0) | (x == 0))
            elif rows:
                dropped = f == 0
                assert torch.equal(y.cpu()[dropped], r[dropped])


def test_dropped_infinities_are_zero():
    import paper_2511_20564_b200 as E
    x = torch.full((64, 128), float("inf"), dtype=BF16, device="cuda")
    x[::2] = float("nan")
    f = R.factors(64, 128, 0.5, 11)
    y = E.dropout(x, E.Dropout(0.5, 11)).cpu()
    assert (y[f == 0] == 0).all() and not torch.isfinite(y[f != 0]).any()


class Norm:
    def __init__(self, rows, dim, dtype, residual, p, mean=0.0, spread=1.0, gains=True, sum_grad=False, seed=0):
        self.x, self.dy = _randn(rows, dim, seed=seed + 1, dtype=dtype, mean=mean), _randn(rows, dim, seed=seed + 2, dtype=dtype)
        self.r = (_randn(rows, dim, seed=seed + 3, dtype=dtype) * spread).to(dtype) if residual else None
        self.gain = 1 + 0.2 * torch.randn(dim, generator=torch.Generator().manual_seed(seed + 4)) if gains else None
        self.shift = torch.randn(dim, generator=torch.Generator().manual_seed(seed + 5)) if gains else None
        self.dz = _randn(rows, dim, seed=seed + 6, dtype=dtype) if sum_grad else None
        self.p, self.seed, self.dtype, self.eps = p, 1000 + seed, dtype, 1e-5
        f = R.factors(rows, dim, p, self.seed, 2, 9)
        d = lambda t: None if t is None else t.double()
        self.want = R.norm(d(self.x), d(self.r), f, d(self.gain), d(self.shift), self.eps, dtype, d(self.dy), d(self.dz))

    def run(self, E, place=lambda t: t.cuda(), stream=None, inplace=False):
        c = lambda t: None if t is None else place(t)
        g = lambda t: None if t is None else t.cuda()
        drop = E.Dropout(self.p, self.seed, place=2, step=9) if self.p else None
        x, r, dy, dz = c(self.x), c(self.r), c(self.dy), c(self.dz)
        y, z, stats = E.layer_norm_forward(x, g(self.gain), g(self.shift), residual=r, drop=drop, eps=self.eps, keep_sum=True,
                                           Y=c(torch.full_like(self.x, 7)), Z=c(torch.full_like(self.x, 7)), stream=stream)
        both = dict(dX=dy, dR=dz) if inplace else dict(dX=c(torch.full_like(self.x, 7)))
        dx, dr, dgain, dshift, _ = E.layer_norm_backward(dy, x, stats, g(self.gain), residual=r, drop=drop, dZ=dz, stream=stream, **both)
        assert (dr is None) == (r is None and not inplace)
        got = dict(y=y, z=z, m=stats[:, :1], s=stats[:, 1:], dx=dx, dgain=dgain, dshift=dshift)
        return {**got, "dr": dr} if dr is not None else got

    def check(self, got):
        for name, t in got.items():
            _held(t, *self.want[name], name)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [4, 8, 12, 16, 36, 40, 64, 72, 128, 256, 264, 320, 512, 516, 1000, 1024, 1032, 2048, 2056, 4096, 8192])
def test_norm_of_every_width(dtype, dim):
    import paper_2511_20564_b200 as E
    if dtype == BF16 and dim % 8:
        pytest.skip("rows of bf16 come in units of 8")
    for rows, residual, p in ((5, False, 0.0), (67, True, 0.25)):
        n = Norm(rows, dim, dtype, residual, p, sum_grad=residual, seed=dim)
        n.check(n.run(E))
        n.check(n.run(E, place=lambda t: _wide(t, 16 // t.element_size())))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [0, 1, 2, 31, 64, 65, 40_000])
def test_norm_of_every_length(dtype, rows):
    import paper_2511_20564_b200 as E
    for residual, p, gains in ((True, 0.1, True), (False, 0.5, False), (True, 0.0, False)):
        n = Norm(rows, 64, dtype, residual, p, gains=gains, seed=rows)
        n.check(n.run(E))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_where_a_difference_of_sums_would_fail(dtype):
    """A mean far from zero, next to no spread, one value that towers above the rest, constant rows."""
    import paper_2511_20564_b200 as E
    n = Norm(50, 320, dtype, True, 0.0, mean=200.0, spread=0.25)
    n.check(n.run(E))
    x = torch.zeros(4, 256, dtype=dtype)
    x[0], x[1, 0], x[2], x[3, 5] = 3.0, 1000.0, -1e-3, -50.0
    got = E.layer_norm_forward(x.cuda(), eps=1e-5)[0]
    want = R.norm(x.double(), None, torch.ones(4, 256), None, None, 1e-5, dtype)
    _held(got, *want["y"], "y")


def test_norm_in_place_and_on_a_stream():
    import paper_2511_20564_b200 as E
    for dtype in (BF16, F32):
        n = Norm(300, 512, dtype, True, 0.2, sum_grad=True)
        n.check(n.run(E, inplace=True))
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        got = n.run(E, stream=stream)
        stream.synchronize()
        n.check(got)
        x = n.x.cuda()
        y, z, _ = E.layer_norm_forward(x, n.gain.cuda(), n.shift.cuda(), residual=n.r.cuda(), drop=E.Dropout(0.2, n.seed, place=2, step=9), Y=x)
        assert y is x and z is None
        _held(y, *n.want["y"], "y")


def test_norm_repeats_bit_for_bit():
    import paper_2511_20564_b200 as E
    n = Norm(20_000, 320, BF16, True, 0.1)
    first = n.run(E)
    for _ in range(5):
        for name, t in n.run(E).items():
            assert torch.equal(t, first[name]), name


def test_captured_steps_drop_by_the_step_on_the_device():
    import paper_2511_20564_b200 as E
    x, r = _randn(100, 256, seed=1, dtype=BF16).cuda(), _randn(100, 256, seed=2, dtype=BF16).cuda()
    dy = _randn(100, 256, seed=3, dtype=BF16).cuda()
    offset = torch.zeros(1, dtype=torch.int32, device="cuda")
    plan = E.Dropout(0.3, 99, place=1, step=4, step_dev=offset)

    def step():
        y, _, stats = E.layer_norm_forward(x, residual=r, drop=plan)
        return [y, E.dropout(x, plan)] + list(E.layer_norm_backward(dy, x, stats, residual=r, drop=plan)[:4])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for k in (0, 5, -4):
        offset.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        f = R.factors(100, 256, 0.3, 99, 1, 4 + k)
        want = R.norm(x.double().cpu(), r.double().cpu(), f, None, None, 1e-5, BF16, dy.double().cpu())
        for t, name in zip(outs, ("y", None, "dx", "dr", "dgain", "dshift")):
            if name:
                _held(t, *want[name], (k, name))
        assert torch.equal(outs[1].cpu() == 0, (f == 0) | (x.cpu() == 0))
