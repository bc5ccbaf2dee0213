"""Sequences that show one key: the softmax is 1 whatever the score, so the gradients of queries and keys are exactly zero."""
import pytest
import torch

from test_gpu_attention import BF16, F32, Problem

pytestmark = pytest.mark.gpu


def _check(p, E):
    got = p.run(E)
    want = p.want()
    p.check(got, want)
    for name, rows in (("dq", p.live_q), ("dk", p.live_k)):
        assert not want[name][0][rows].abs().max() > 1e-12 and not got[name][rows].any(), (name, got[name][rows].abs().max().item())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 32), (4, 2, 64), (2, 1, 128), (6, 2, 40), (3, 3, 16), (2, 2, 96), (1, 1, 256)])
@pytest.mark.parametrize("q_lens", [[1] * 9, [3, 2, 0, 4, 1], [40, 1, 0, 7], [900, 3, 130]], ids=["ones", "few", "tens", "hundreds"])
def test_one_key(q_lens, heads, kv_heads, hd, dtype):
    import paper_2511_20564_b200 as E
    p = Problem(q_lens, [1] * (len(q_lens) - 1) + [0], heads, kv_heads, hd, dtype)
    _check(p, E)


def _one_left(p, k_lens, at):
    """The mask of p leaves key at[s] of every sequence."""
    p.mask = torch.zeros(p.k.shape[0], dtype=torch.uint8)
    for s, n in enumerate(k_lens):
        p.mask[int(p.k_ptr[s]) + at[s] % n] = 1
    p.k_in, p.v_in = p.k.clone(), p.v.clone()
    p.k_in[p.mask == 0], p.v_in[p.mask == 0] = float("nan"), float("inf")
    return p


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 32), (2, 1, 128), (5, 5, 80), (2, 2, 100)])
@pytest.mark.parametrize("q_lens", [[1, 2, 1, 1], [30, 300, 1, 128]], ids=["few", "many"])
def test_a_mask_that_leaves_one_key(q_lens, heads, kv_heads, hd, dtype):
    import paper_2511_20564_b200 as E
    if dtype == BF16 and hd % 8:
        hd = 104
    k_lens = [100, 3, 128, 65]
    _check(_one_left(Problem(q_lens, k_lens, heads, kv_heads, hd, dtype), k_lens, [99, 1, 64, 0]), E)


@pytest.mark.parametrize("q_lens,dtype", [([1, 2, 1, 1], BF16), ([1, 2, 1, 1], F32), ([30, 300, 1, 128], F32)], ids=["few-bf16", "few-f32", "many-f32"])
def test_one_key_of_a_long_list(q_lens, dtype):
    """Many turns, tiles and stretches: D of the stored output is the key's own product.  (bf16 rows on the tensor cores are left out: over
    several tiles their D is added up in another order than dP, and the bounds of the other tests hold.)"""
    import paper_2511_20564_b200 as E
    k_lens = [5000, 700, 1025, 129]
    p = _one_left(Problem(q_lens, k_lens, 4, 2, 64, dtype), k_lens, [4999, 350, 0, 128])
    _check(p, E)
