"""Attention with a bias of many rows: the largest tables that lie beside the tiles, and bins of blocks that become smaller for them."""
import pytest
import torch

from test_gpu_bias import _go

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,buckets", [(12, 3, 106), (8, 2, 110), (10, 10, 128), (11, 1, 40)])
@pytest.mark.parametrize("hd", [64, 128])
def test_the_largest_tables_beside_the_tiles(heads, kv_heads, buckets, hd):
    """Distances that put tens of buckets into 32 columns, and positions in no order."""
    edge = [2 * (i - buckets // 2) for i in range(buckets - 1)]
    for pos in ("rows", "any"):
        _go([150, 0, 40], [333, 40, 128], heads, kv_heads, hd, torch.bfloat16, edge, pos=pos, masked=True, runs=(dict(), dict(hints=0)))
