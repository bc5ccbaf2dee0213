"""Attention with a bias of few rows: numbers of key heads that leave a warp's last group of heads short."""
import numpy as np
import pytest
import torch

from test_gpu_bias import BOTH, _go

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
HEADS = [(3, 3, 32), (6, 3, 32), (6, 6, 16), (5, 5, 16), (7, 7, 8), (3, 3, 8), (3, 3, 64), (11, 11, 8), (3, 3, 128)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,hd", HEADS)
@pytest.mark.parametrize("pos", ["times", "any", "far"])
def test_groups_of_heads_that_are_not_full(dtype, heads, kv_heads, hd, pos):
    rng = np.random.default_rng(hd)
    for lens in (([1] * 30, rng.integers(0, 130, 30)), ([2, 1, 0, 1], [60, 7, 90, 333]), ([3, 5, 1], [4, 30, 25])):
        _go(*lens, heads, kv_heads, hd, dtype, BOTH, pos=pos, masked=True, runs=(dict(), dict(hints=0)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,hd", HEADS[:4])
def test_long_histories_of_such_heads(dtype, heads, kv_heads, hd):
    _go([1, 2], [5000, 2500], heads, kv_heads, hd, dtype, BOTH, pos="times", runs=(dict(), dict(hints=0)))
