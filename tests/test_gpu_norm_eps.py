"""Norms of heads with eps = 0, and of heads whose squares are small."""
import pytest
import torch

import fusion_oracle as F

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
E24 = 2.0 ** -24


def _randn(*shape, seed, dtype):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,hd", [(1, 1, 8), (130, 3, 40), (257, 2, 64), (19, 7, 96), (33, 1, 256)])
def test_gains_with_eps_zero(rows, heads, hd, dtype):
    """Threads without a row add nothing to the gains' gradients: the norm of their zeros has no inverse."""
    import paper_2511_20564_b200 as E
    x, g = _randn(rows, heads * hd, seed=1, dtype=dtype), _randn(rows, heads * hd, seed=2, dtype=dtype)
    w = 1 + 0.2 * _randn(hd, seed=3, dtype=F32)
    dq, dk, dwq, dwk, _ = E.qk_norm_rotary_backward(g.cuda(), g.cuda(), x.cuda(), x.cuda(), heads, heads, w.cuda(), w.cuda(), eps=0.0)
    none = torch.empty(0, dtype=torch.float64)
    dx, dw, dx_terms, dw_terms = F.norm_rotary_backward(g.double(), x.double(), heads, w.double(), 0.0, none, torch.zeros(rows))
    norm = (hd + 8) * E24             # relative error of 1 / rms and of a mean over a head in 32 bits
    for got in (dq, dk):
        assert ((got.double().cpu() - dx).abs() <= F.HALF[dtype] * dx.abs() + 3 * norm * dx_terms).all()
    for got in (dwq, dwk):
        assert ((got.double().cpu() - dw).abs() <= (3 * norm + (rows * heads + 600) * E24) * dw_terms).all()
