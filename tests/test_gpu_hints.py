"""Longest sequences that the caller names too small: gradients as accurate as with right ones."""
import pytest
import torch

import fusion_oracle as F

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
# A value rounded to nearest is off by at most half a step, evenly spread: in the mean by 1 / sqrt(3) of that, and relative to the value at
# most by that share of 2^-8 (a matrix's error relative to its norm, over many elements); 5 % for the sample and for fp32 sums.
ROUNDED = 1.05 * F.HALF[BF16] / 3 ** 0.5


@pytest.mark.parametrize("q_len,heads,kv_heads,hd", [(1, 4, 4, 32), (2, 4, 2, 64), (3, 2, 2, 128)])
@pytest.mark.parametrize("mk", [1, 3, 0])
def test_a_hint_that_is_too_small_costs_no_accuracy(mk, q_len, heads, kv_heads, hd):
    """Keys that are alike but for an eighth: what D lacks by the rounding of the 16-bit outputs, 1.5e-3 of it, would meet the sum of all
    p k in dQ, eight times as large as what the keys differ by."""
    import paper_2511_20564_b200 as E
    gen = torch.Generator().manual_seed(11)
    n, k_len = 40, 700
    q_ptr, k_ptr = torch.arange(n + 1) * q_len, torch.arange(n + 1) * k_len
    make = lambda rows, w: torch.randn(rows, w, generator=gen)
    q, g = make(n * q_len, heads * hd).to(BF16), make(n * q_len, heads * hd).to(BF16)
    k, v = (1 + 0.125 * make(n * k_len, kv_heads * hd)).to(BF16), make(n * k_len, kv_heads * hd).to(BF16)
    seqs = E.Sequences(q_ptr.cuda(), k_ptr.cuda(), q_len, mk)
    cu = [t.cuda() for t in (q, k, v, g)]
    out, lse, _ = E.cross_attention_forward(*cu[:3], seqs, heads, kv_heads, hd ** -0.5)
    dq = E.cross_attention_backward(cu[3], *cu[:3], out, lse, seqs, heads, kv_heads, hd ** -0.5)[0]
    want = F.attention(q.double(), k.double(), v.double(), q_ptr, k_ptr, heads, kv_heads, hd ** -0.5, None, g.double(), BF16)["dq"][0]
    err = ((dq.double().cpu() - want).norm() / want.norm()).item()
    assert err <= ROUNDED, err
