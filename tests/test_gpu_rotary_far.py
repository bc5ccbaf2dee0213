"""Rotary angles of far positions and of tables with large frequencies, against exact integers."""
from fractions import Fraction
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
# 1 / (2 pi) to 60 digits
TURNS = Fraction(159154943091895335768883763372514362034459645740456448747667, 10 ** 60)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
def test_far_positions(inter, dtype):
    """Position times frequency modulo a turn to 2^-32 of a turn: sine and cosine, and the sums of two products, are what the results are
    off by (2^-20 for 16-bit results with the angle's 23 bits, 2^-21 for 32-bit ones), however many turns lie behind."""
    import paper_2511_20564_b200 as E
    hd, rows = 64, 97
    gen = torch.Generator().manual_seed(7)
    x = torch.randn(rows, hd, generator=gen).to(dtype)
    pos = torch.randint(-(1 << 31), 1 << 31, (rows,), generator=gen, dtype=torch.int64)
    pos[:4] = torch.tensor([(1 << 31) - 1, -(1 << 31), 40_000_003, 0])
    freqs = torch.cat([10_000.0 ** (-torch.arange(16, dtype=torch.float64) / 16), 1000 * torch.rand(14, generator=gen, dtype=torch.float64),
                       torch.tensor([-0.7, 12345.678], dtype=torch.float64)])
    turns = torch.tensor([[float(Fraction(f) * p * TURNS % 1) for f in freqs.tolist()] for p in pos.tolist()], dtype=torch.float64)
    c, s = torch.cos(2 * math.pi * turns), torch.sin(2 * math.pi * turns)
    i = torch.arange(hd // 2)
    a, b = (2 * i, 2 * i + 1) if inter else (i, i + hd // 2)
    xd, want, size = x.double(), torch.empty(rows, hd, dtype=torch.float64), torch.empty(rows, hd, dtype=torch.float64)
    want[:, a], want[:, b] = xd[:, a] * c - xd[:, b] * s, xd[:, b] * c + xd[:, a] * s
    size[:, a] = size[:, b] = xd[:, a].abs() + xd[:, b].abs()
    got = E.rotary(x.cuda(), 1, freqs.cuda(), pos.to(torch.int32).cuda(), interleaved=inter).double().cpu()
    trig, half = (2.0 ** -20, 2.0 ** -8) if dtype == BF16 else (2.0 ** -21, 2.0 ** -24)
    assert ((got - want).abs() <= half * want.abs() + (trig + 4 * 2.0 ** -24) * size).all(), ((got - want).abs() / size).max().item()
