"""Attention: rows of hidden keys get zeros where visible keys and values of their sequence hold infinities and NaN."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 32), (2, 1, 64), (2, 2, 256), (8, 2, 128)])
@pytest.mark.parametrize("q_lens", [[1, 1, 1, 1], [3, 2, 4, 3], [20, 70, 9, 300]], ids=["ones", "few", "many"])
@pytest.mark.parametrize("k_lens", [[90, 3, 200, 64], [4, 3, 9, 2]], ids=["turns", "turn"])
@pytest.mark.parametrize("hints", [True, False])
@pytest.mark.parametrize("where", ["keys", "values"])
def test_hidden_keys_get_zeros_beside_keys_that_overflowed(where, hints, k_lens, q_lens, heads, kv_heads, hd, dtype):
    import paper_2511_20564_b200 as E
    gen = torch.Generator().manual_seed(5)
    q_ptr, k_ptr = (torch.tensor([0] + l).cumsum(0) for l in (q_lens, k_lens))
    make = lambda rows, h: torch.randn(int(rows), h * hd, generator=gen).to(dtype)
    q, g, k, v = make(q_ptr[-1], heads), make(q_ptr[-1], heads), make(k_ptr[-1], kv_heads), make(k_ptr[-1], kv_heads)
    mask = (torch.rand(int(k_ptr[-1]), generator=gen) > 0.4).to(torch.uint8)
    hidden = mask == 0
    seen = (~hidden).nonzero()[:, 0]
    t = k if where == "keys" else v
    t[seen[::3], ::5], t[seen[1::4], 1::4] = INF, NAN
    longest = (max(q_lens), max(k_lens)) if hints else (1, 1)
    seqs = E.Sequences(q_ptr.cuda(), k_ptr.cuda(), *longest, k_mask=mask.cuda())
    args = q.cuda(), k.cuda(), v.cuda()
    out, lse, _ = E.cross_attention_forward(*args, seqs, heads, kv_heads, hd ** -0.5)
    _, dk, dv, _ = E.cross_attention_backward(g.cuda(), *args, out, lse, seqs, heads, kv_heads, hd ** -0.5)
    gone = hidden.cuda()
    assert dk[~gone].isnan().any()                       # (dV goes by p and dOut alone: values do not reach it)
    assert (dk[gone] == 0).all() and (dv[gone] == 0).all()
