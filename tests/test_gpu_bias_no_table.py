"""Attention with a bias: whether the table's gradient is asked for changes nothing in the others."""
import pytest
import torch

from test_gpu_bias import BOTH, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 32), (4, 2, 64), (8, 2, 128), (6, 2, 40)])
@pytest.mark.parametrize("lens", [([1] * 30, [100] * 30), ([3, 1, 2, 4], [60, 7, 90, 300]), ([70, 3, 200], [300, 40, 700]), ([2, 1], [4000, 100])],
                         ids=["ones", "few", "many", "long"])
def test_gradients_are_the_same_without_the_tables(lens, heads, kv_heads, hd, dtype):
    import paper_2511_20564_b200 as E
    p = Problem(*lens, heads, kv_heads, hd, dtype, BOTH, masked=True, seed=hd, mean=1.0)
    res = p.run(E)
    args = [t.cuda() for t in (p.g_in, p.q_in, p.k_in, p.v_in)]
    got = E.biased_attention_backward(*args, res["out"], res["lse"], p.seqs(E), p.bias(E), heads, kv_heads, p.scale, table_grad=False)
    assert got[3] is None
    for t, name, live in ((got[0], "dq", p.live_q), (got[1], "dk", p.live_k), (got[2], "dv", p.live_k)):
        assert torch.equal(t[live], res[name][live]), name
