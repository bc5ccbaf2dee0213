"""How far bf16 results are off in the mean: errors relative to a result's norm.  The element-wise bounds of the other tests are worst cases,
too wide to see a correction that is missing."""
import pytest
import torch

import fusion_oracle as F
from test_gpu_attention import BF16, HEADS, LENGTHS, Problem

pytestmark = pytest.mark.gpu

# A value rounded to nearest is off by at most half a step, evenly spread: its error has a root mean square of 1 / sqrt(3) of that, relative
# to a value at most 2^-8 / sqrt(3) = 2.26e-3 (1.5e-3 for spread mantissas).  Sums of independently rounded terms are off by no more
# than that share of the norm of what they sum; independent errors add in squares, so adding them up plainly leaves room.
U = F.HALF[BF16] / 3 ** 0.5


def _off(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("masked", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("heads,kv_heads,hd", HEADS)
@pytest.mark.parametrize("lengths", [name for name in LENGTHS if name != "ones"])
def test_errors_of_random_inputs(lengths, heads, kv_heads, hd, masked):
    """out, dV: p and the result are rounded.  dQ: D from the stored out and the result (dS as two values keeps 16 bits).  dK: dS, D and the
    result.  A gradient that is 3 % too large, or a product with the wrong sign, is beyond all of them."""
    import paper_2511_20564_b200 as E
    p = Problem(*LENGTHS[lengths], heads, kv_heads, hd, BF16, masked, seed=3)
    got, want = p.run(E), p.want()
    for name, steps in (("out", 2), ("dv", 2), ("dq", 2), ("dk", 3)):
        rows = p.live_k if name in ("dk", "dv") else p.live_q
        assert _off(got[name][rows], want[name][0][rows]) <= 1.05 * steps * U, name


def _alike(rows, width, gen):
    """Keys that differ by an eighth of what they have in common: an error of all dS of a row alike, or the roundings of dS one by one, come
    out eight times as large in dQ = sum dS k, whose common part is sum dS = 0."""
    return (1 + 0.125 * torch.randn(rows, width, generator=gen)).to(BF16)


@pytest.mark.parametrize("n_seq,q_len,k_len,heads,kv_heads,hd", [
    (600, 1, 90, 4, 4, 32), (300, 2, 200, 4, 4, 64), (9, 1, 3001, 4, 2, 64), (2, 1, 24000, 2, 2, 128), (1, 2, 9000, 2, 1, 40),
    (3, 3, 5000, 3, 3, 96), (2, 1, 7000, 8, 2, 256), (40, 4, 500, 1, 1, 128)])
def test_streamed_dq_without_what_the_stored_outputs_lack(n_seq, q_len, k_len, heads, kv_heads, hd):
    """One warp per sequence, several, and stretches of the keys that are joined: D of the 16-bit outputs is off by 1.5e-3 of itself, which
    is taken out of dQ; without that, or with it taken the wrong way, dQ here is off by 1e-2.  With it the result's rounding is left,
    and fp32 sums."""
    import paper_2511_20564_b200 as E
    gen = torch.Generator().manual_seed(k_len)
    make = lambda rows, h: torch.randn(rows, h * hd, generator=gen).to(BF16)
    q, g, v = make(n_seq * q_len, heads), make(n_seq * q_len, heads), make(n_seq * k_len, kv_heads)
    k = _alike(n_seq * k_len, kv_heads * hd, gen)
    q_ptr, k_ptr = torch.arange(n_seq + 1) * q_len, torch.arange(n_seq + 1) * k_len
    seqs = E.Sequences(q_ptr.cuda(), k_ptr.cuda(), q_len, k_len)
    cu = [t.cuda() for t in (q, k, v, g)]
    out, lse, _ = E.cross_attention_forward(*cu[:3], seqs, heads, kv_heads, hd ** -0.5)
    dq = E.cross_attention_backward(cu[3], *cu[:3], out, lse, seqs, heads, kv_heads, hd ** -0.5)[0]
    want = F.attention(q.double(), k.double(), v.double(), q_ptr, k_ptr, heads, kv_heads, hd ** -0.5, None, g.double(), BF16)["dq"][0]
    assert _off(dq, want) <= 1.05 * U


@pytest.mark.parametrize("q_len,k_len,heads,kv_heads,hd", [(200, 256, 2, 2, 64), (130, 512, 4, 2, 128), (64, 128, 2, 1, 96), (300, 1024, 3, 3, 40)])
def test_tile_dq_with_ds_of_two_values(q_len, k_len, heads, kv_heads, hd):
    """Queries of zero make p = 1 / n exactly, values of -1, 0, 1 make out and D exact: what dS loses as operands of the tensor cores is
    left, one rounding to bf16 1.5e-3 of it and 1.2e-2 of dQ for these keys, two values 2^-8 of that."""
    import paper_2511_20564_b200 as E
    gen, n_seq = torch.Generator().manual_seed(hd), 3
    q = torch.zeros(n_seq * q_len, heads * hd, dtype=BF16)
    g = torch.randn(n_seq * q_len, heads * hd, generator=gen).to(BF16)
    v = torch.randint(-1, 2, (n_seq * k_len, kv_heads * hd), generator=gen).to(BF16)
    k = _alike(n_seq * k_len, kv_heads * hd, gen)
    q_ptr, k_ptr = torch.arange(n_seq + 1) * q_len, torch.arange(n_seq + 1) * k_len
    seqs = E.Sequences(q_ptr.cuda(), k_ptr.cuda(), q_len, k_len)
    cu = [t.cuda() for t in (q, k, v, g)]
    out, lse, _ = E.cross_attention_forward(*cu[:3], seqs, heads, kv_heads, 1.0)
    want = F.attention(q.double(), k.double(), v.double(), q_ptr, k_ptr, heads, kv_heads, 1.0, None, g.double(), BF16)
    exact = (want["out"][0] * k_len).round() / k_len          # a whole number over k_len, as 64 bits have it but for 1e-16
    assert (exact - want["out"][0]).abs().max() <= 1e-14 and torch.equal(out.double().cpu(), exact)
    dq = E.cross_attention_backward(cu[3], *cu[:3], out, lse, seqs, heads, kv_heads, 1.0)[0]
    assert _off(dq, want["dq"][0]) <= 1.05 * U
