"""The 64-bit form of attention with a bias: gradients against differences, buckets and edges by their definition."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import bias_oracle as F
from paper_2511_20564_b200 import binding as B


def _problem(hidden=False):
    gen = torch.Generator().manual_seed(8)
    rnd = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    q_ptr, k_ptr = torch.tensor([0, 3, 3, 5]), torch.tensor([0, 4, 7, 12])
    edge = torch.tensor([-5, -2, 0, 3], dtype=torch.int32)
    table = rnd(5, 4)
    if hidden:
        table[1, 2] = -math.inf
        table[2, 0] = -1e30
    pos_q, pos_k = torch.tensor([4, 9, 2, 7, 1]), torch.randint(0, 10, (12,), generator=gen)
    return rnd(5, 8), rnd(12, 4), rnd(12, 4), rnd(5, 8), table, dict(q_ptr=q_ptr, k_ptr=k_ptr, heads=4, kv_heads=2, scale=0.7, edge=edge, pos_q=pos_q, pos_k=pos_k)


@pytest.mark.parametrize("hidden", [False, True])
def test_gradients_against_differences(hidden):
    q, k, v, g, table, kw = _problem(hidden)
    loss = lambda q, k, v, table: (F.attention(q, k, v, table=table, **kw)["out"][0] * g).sum()
    got = F.attention(q, k, v, table=table, dout=g, **kw)
    args = [q, k, v, table]
    for i, name in enumerate(("dq", "dk", "dv", "dtable")):
        for at in np.ndindex(*args[i].shape):
            if name == "dtable" and args[i][at] <= F.HIDES:
                assert got[name][0][at] == 0
                continue
            ends = []
            for step in (1e-6, -1e-6):
                moved = [a.clone() for a in args]
                moved[i][at] += step
                ends.append(loss(*moved))
            assert abs(got[name][0][at] - (ends[0] - ends[1]) / 2e-6) < 1e-6, (name, at)


def test_a_row_of_hidden_buckets_is_empty():
    q, k, v, g, table, kw = _problem()
    table[:, 1] = -1e30
    got = F.attention(q, k, v, table=table, dout=g, **kw)
    assert (got["out"][0][:3, 2:4] == 0).all() and torch.isinf(got["lse"][0][:, 1]).all() and (got["dq"][0][:, 2:4] == 0).all()


@pytest.mark.parametrize("buckets,far,both", [(1, 5, False), (1, 5, True), (2, 1, True), (16, 128, True), (32, 100_000, False), (32, 128, False), (63, 7, True),
                                              (64, 1 << 30, True), (128, 1 << 30, False), (3, 2, False), (60, 20_000, True)])
def test_edges(buckets, far, both):
    n = max(2 * buckets - 2 if both else buckets - 1, 0)
    got = np.full(n + 1, 77, dtype=np.int32)
    assert B.lib().e2egrec_relative_edges(buckets, far, int(both), got.ctypes.data) == 0
    assert got[n] == 77 and got[:n].tolist() == F.edges(buckets, far, both) and (np.diff(got[:n]) > 0).all()


def test_edges_refusals():
    f, out = B.lib().e2egrec_relative_edges, (C.c_int32 * 300)()
    assert f(0, 5, 0, out) == -2 and f(4, 0, 0, out) == -2 and f(4, (1 << 30) + 1, 0, out) == -2 and f(129, 5, 0, out) == -6 and f(65, 5, 1, out) == -6
    assert f(4, 5, 0, None) == -1 and f(1, 5, 0, None) == 0


def test_buckets_of_the_usual_form():
    """Powers of the ratio that are whole numbers begin their bucket: 16 exact, then 16 by the logarithm up to 16 * 2^4."""
    edge = torch.tensor(F.edges(32, 256))
    past = lambda d: F.buckets(edge, torch.tensor([0]), torch.tensor([-d])).item()
    assert [31 - past(d) for d in (0, 1, 15, 16, 31, 32, 63, 64, 127, 128, 255, 256, 10_000)] == [0, 1, 15, 16, 19, 20, 23, 24, 27, 28, 31, 31, 31]
