"""Attention with a bias: what hidden keys get where visible keys and values, or queries and gradients, hold infinities and NaN."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 32), (2, 1, 64), (2, 2, 256), (8, 2, 128)])
@pytest.mark.parametrize("q_lens", [[1, 1, 1, 1], [3, 2, 4, 3], [20, 70, 9, 300]], ids=["ones", "few", "many"])
@pytest.mark.parametrize("hints", [True, False])
@pytest.mark.parametrize("where", ["keys", "values", "rows"])
@pytest.mark.parametrize("table_grad", [True, False])
def test_hidden_keys_stay_at_zero(table_grad, where, hints, q_lens, heads, kv_heads, hd, dtype):
    """Rows of hidden keys get zeros, and a bucket that only hidden keys are in has no gradient."""
    import paper_2511_20564_b200 as E
    gen = torch.Generator().manual_seed(3)
    k_lens = [90, 3, 200, 64]
    q_ptr, k_ptr = (torch.tensor([0] + l).cumsum(0) for l in (q_lens, k_lens))
    make = lambda rows, h: torch.randn(int(rows), h * hd, generator=gen).to(dtype)
    q, g, k, v = make(q_ptr[-1], heads), make(q_ptr[-1], heads), make(k_ptr[-1], kv_heads), make(k_ptr[-1], kv_heads)
    mask = (torch.rand(int(k_ptr[-1]), generator=gen) > 0.4).to(torch.uint8)
    hidden = mask == 0
    seen = (~hidden).nonzero()[:, 0]
    if where == "keys":
        k[seen[::7], ::5], k[seen[3::11], 1::4] = INF, NAN
    if where == "values":
        v[seen[::7], ::5], v[seen[3::11], 1::4] = INF, NAN
    # distances: 0 .. 9 of visible keys, 1000 .. 1009 of hidden ones, behind the last edge
    pos_q = torch.zeros(int(q_ptr[-1]), dtype=torch.int32)
    pos_k = (torch.arange(int(k_ptr[-1])) % 10 + hidden * 1000).to(torch.int32)
    edges = torch.tensor([2, 5, 700, 900], dtype=torch.int32)
    bias = E.RelativeBias(torch.randn(5, heads, generator=gen).cuda(), edges.cuda(), pos_q.cuda(), pos_k.cuda())
    longest = (max(q_lens), max(k_lens)) if hints else (1, 1)
    seqs = E.Sequences(q_ptr.cuda(), k_ptr.cuda(), *longest, k_mask=mask.cuda())
    out, lse, _ = E.biased_attention_forward(q.cuda(), k.cuda(), v.cuda(), seqs, bias, heads, kv_heads, hd ** -0.5)
    if where == "rows":
        q, g = q.clone(), g.clone()
        q[::2, ::5], g[::3, ::7], g[1::3, 1::4] = INF, INF, NAN
    _, dk, dv, dtable, _ = E.biased_attention_backward(g.cuda(), q.cuda(), k.cuda(), v.cuda(), out, lse, seqs, bias, heads, kv_heads, hd ** -0.5,
                                                       table_grad=table_grad)
    gone = hidden.cuda()
    assert hidden.any() and not dk[gone].any() and not dv[gone].any()
    if table_grad:
        assert not dtable[3:].any()
