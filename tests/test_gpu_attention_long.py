"""Rows over long lists of keys on the tensor cores: dQ shrinks with the number of keys, what D of the 16-bit outputs lacks does not."""
import pytest
import torch

import fusion_oracle as F
from test_gpu_attention import BF16
from test_gpu_attention_norms import U, _off

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("masked", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("q_lens,k_lens,heads,kv_heads,hd", [
    ([40, 3], [26000, 700], 2, 1, 16), ([30], [20000], 4, 2, 64), ([9, 0, 9], [16001, 40, 127], 16, 4, 40), ([20], [30000], 2, 2, 128),
    ([300, 5], [9000, 2049], 1, 1, 32), ([7], [12345], 6, 2, 96), ([130, 2, 260], [2048, 5000, 3000], 2, 2, 64)])
def test_dq_of_long_lists(q_lens, k_lens, heads, kv_heads, hd, masked):
    """Values that are not spread around zero, so that D is as large as dP.  The roundings of the 16-bit outputs in it meet sum p k, which goes to
    scale q, while dQ goes down with the root of the number of keys: 9e-3 of it over 26 000 keys.  What is left may be the result's
    rounding and, in sequences of up to 32 head_dim keys, as much again.  dK and dV as in sequences of any length."""
    import paper_2511_20564_b200 as E
    gen = torch.Generator().manual_seed(hd)
    ptr = lambda l: torch.tensor([0] + l).cumsum(0)
    q_ptr, k_ptr = ptr(q_lens), ptr(k_lens)
    make = lambda rows, h, mean=0.0: (torch.randn(int(rows), h * hd, generator=gen) + mean).to(BF16)
    q, g, k, v = make(q_ptr[-1], heads), make(q_ptr[-1], heads), make(k_ptr[-1], kv_heads), make(k_ptr[-1], kv_heads, 0.25)
    mask = (torch.rand(int(k_ptr[-1]), generator=gen) > 0.1).to(torch.uint8) if masked else None
    want = F.attention(*(t.double() for t in (q, k, v)), q_ptr, k_ptr, heads, kv_heads, hd ** -0.5, mask, g.double(), BF16, True)
    cu = [t.cuda() for t in (q, k, v, g)]
    for hints in ((max(q_lens), max(k_lens)), (0, 0)):
        seqs = E.Sequences(q_ptr.cuda(), k_ptr.cuda(), *hints, k_mask=None if mask is None else mask.cuda())
        out, lse, _ = E.cross_attention_forward(*cu[:3], seqs, heads, kv_heads, hd ** -0.5)
        dq, dk, dv, _ = E.cross_attention_backward(cu[3], *cu[:3], out, lse, seqs, heads, kv_heads, hd ** -0.5)
        for s, n in enumerate(k_lens):
            rows, keys = slice(q_ptr[s], q_ptr[s + 1]), slice(k_ptr[s], k_ptr[s + 1])
            if not q_lens[s]:
                continue
            # (5 %: samples of some hundred values, fp32 sums of as many terms as there are keys)
            assert _off(dq[rows], want["dq"][0][rows]) <= 1.05 * (1 if n > 32 * hd else 2) * U, (hints, s)
            assert _off(dk[keys], want["dk"][0][keys]) <= 1.05 * 3 * U and _off(dv[keys], want["dv"][0][keys]) <= 1.05 * 2 * U, (hints, s)
