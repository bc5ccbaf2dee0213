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


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 32), (2, 1, 64), (2, 2, 256)])
@pytest.mark.parametrize("q_lens", [[1, 1, 1, 1], [3, 2, 4, 3], [20, 70, 9, 300]], ids=["ones", "few", "many"])
@pytest.mark.parametrize("hints", [True, False])
def test_hidden_keys_get_zeros_beside_rows_that_overflowed(hints, q_lens, heads, kv_heads, hd, dtype):
    """Queries and gradients that hold infinities and NaN (a step whose loss overflowed): rows of hidden keys still get zeros."""
    import paper_2511_20564_b200 as E
    gen = torch.Generator().manual_seed(3)
    k_lens = [90, 3, 200, 64]
    q_ptr, k_ptr = (torch.tensor([0] + l).cumsum(0) for l in (q_lens, k_lens))
    make = lambda rows, h: torch.randn(int(rows), h * hd, generator=gen).to(dtype)
    q, g, k, v = make(q_ptr[-1], heads), make(q_ptr[-1], heads), make(k_ptr[-1], kv_heads), make(k_ptr[-1], kv_heads)
    mask = (torch.rand(int(k_ptr[-1]), generator=gen) > 0.4).to(torch.uint8)
    hidden = mask == 0
    hidden_dev = hidden.cuda()
    longest = (max(q_lens), max(k_lens)) if hints else (1, 1)
    seqs = E.Sequences(q_ptr.cuda(), k_ptr.cuda(), *longest, k_mask=mask.cuda())
    out, lse, _ = E.cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), seqs, heads, kv_heads, hd ** -0.5)
    q, g = q.clone(), g.clone()
    q[::2, ::5], g[::3, ::7], g[1::3, 1::4] = INF, INF, NAN
    _, dk, dv, _ = E.cross_attention_backward(g.cuda(), q.cuda(), k.cuda(), v.cuda(), out, lse, seqs, heads, kv_heads, hd ** -0.5)
    assert hidden.any() and not dk[hidden_dev].any() and not dv[hidden_dev].any()
