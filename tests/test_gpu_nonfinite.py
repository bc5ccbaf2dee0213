"""Infinities and NaN beside what a call may not let them reach."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("hd,rot,inter", [(40, 20, False), (40, 20, True), (64, 48, False), (64, 42, True), (128, 38, False), (16, 2, False), (96, 0, False)])
def test_what_is_not_rotated_is_copied(hd, rot, inter, dtype):
    """The rest of a head keeps its values whatever stands beside them, signs of zeros too."""
    import paper_2511_20564_b200 as E
    heads, rows = 3, 29
    x = torch.randn(rows, heads * hd, generator=torch.Generator().manual_seed(1)).to(dtype)
    rest = x.view(rows, heads, hd)[..., rot:]
    rest[::2, :, ::3] = INF
    rest[1::4, :, 1::5] = NAN
    rest[:, :, 2::7] = -0.0
    freqs = torch.rand(rot // 2, dtype=torch.float64).cuda() if rot else None
    for inverse in (False, True):
        y = E.rotary(x.cuda(), heads, freqs, None, scale=1.25, interleaved=inter, inverse=inverse).cpu().view(rows, heads, hd)
        same = y[..., rot:].contiguous().view(torch.int16 if dtype == BF16 else torch.int32)
        bits = rest.contiguous().view(same.dtype)
        assert torch.equal(torch.where(rest.isnan(), 0, same), torch.where(rest.isnan(), 0, bits)) and y[..., rot:][rest.isnan()].isnan().all()
        assert y[..., :rot].isfinite().all()
