"""Attention with a bias of many rows: calls back to back, sequences that show one key, and blocks of every size."""
import numpy as np
import pytest
import torch

import bias_oracle as F
from test_gpu_bias import BOTH, Problem, _go

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("heads,kv_heads,hd", [(8, 8, 128), (8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("pos", ["rows", "times"])
def test_calls_back_to_back_repeat(heads, kv_heads, hd, pos):
    """Forty calls on full sequences without a wait between them: the same bits every time."""
    import paper_2511_20564_b200 as E
    p = Problem([1024] * 4, [1024] * 4, heads, kv_heads, hd, BF16, F.edges(32, 1024, True), pos=pos, masked=True, seed=3)
    p.mask[:] = torch.from_numpy((np.random.default_rng(5).random(p.mask.numel()) > 0.1).astype(np.uint8))
    q, k, v, g = (t.cuda() for t in (p.q, p.k, p.v, p.g))
    seqs, bias = p.seqs(E), p.bias(E)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    first = None
    for _ in range(4):
        for _ in range(10):
            out, lse, ws = E.biased_attention_forward(q, k, v, seqs, bias, heads, kv_heads, p.scale, status=status)
            grads = E.biased_attention_backward(g, q, k, v, out, lse, seqs, bias, heads, kv_heads, p.scale, status=status)[:4]
        res = [out[p.live_q], lse[p.live_q], grads[0][p.live_q], grads[1][p.live_k], grads[2][p.live_k], grads[3]]
        assert int(status) == 0 and all(t.isfinite().all() for t in res)
        first = first or [t.clone() for t in res]
        assert all(torch.equal(a, b) for a, b in zip(res, first))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 32), (4, 2, 64), (2, 1, 128), (6, 2, 40), (3, 3, 96)])
@pytest.mark.parametrize("q_lens", [[3, 2, 0, 4, 1], [40, 1, 0, 7, 2], [500, 3, 130, 64, 65]], ids=["few", "tens", "hundreds"])
def test_one_key_has_no_gradient_of_its_scores(q_lens, heads, kv_heads, hd, dtype):
    """The softmax of a lone key is 1 whatever its bias: dQ, dK and the table's gradient are within the bounds of zero, and for bf16 zero itself."""
    import paper_2511_20564_b200 as E
    p = Problem(q_lens, [1] * len(q_lens), heads, kv_heads, hd, dtype, BOTH, pos="any")
    want, got = p.want(), p.run(E)
    p.check(got, want)
    if dtype == BF16:
        assert not got["dq"][p.live_q].any() and not got["dk"][p.live_k].any()


@pytest.mark.parametrize("hd", [16, 24, 40, 56, 72, 88, 104, 128])
@pytest.mark.parametrize("rows", [17, 33, 65, 129])
def test_blocks_of_every_size(rows, hd):
    """Every width of heads, rows and keys that fill one, two, four and eight warps of a block and one row more; groups that divide 8 and that do not."""
    for heads, kv_heads in ((2, 2), (6, 2), (16, 1)):
        _go([rows // (heads // kv_heads) + 1, 0, 5], [rows, 130, 64], heads, kv_heads, hd, BF16, BOTH, pos="times", masked=True, seed=hd)
