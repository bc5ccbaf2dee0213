"""Attention with a bias over so many sequences that a block of the tensor-core kernels takes several units, one after the other."""
import numpy as np
import pytest
import torch

from test_gpu_bias import BOTH, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,hd", [(4, 4, 64), (12, 4, 128), (12, 4, 40), (16, 4, 128), (5, 5, 128)])
@pytest.mark.parametrize("pos", ["any", "times"])
def test_blocks_that_take_unit_after_unit(heads, kv_heads, hd, pos):
    """Some sequences without rows, without keys or hidden altogether between the others; the same bits from run to run."""
    import paper_2511_20564_b200 as E
    rng = np.random.default_rng(hd + heads)
    q_lens, k_lens = rng.integers(20, 41, 700), rng.integers(90, 401, 700)
    q_lens[5::50] = 0
    k_lens[7::60] = 0
    p = Problem(q_lens, k_lens, heads, kv_heads, hd, torch.bfloat16, BOTH, pos=pos, masked=True, seed=hd)
    want = p.want()
    first = p.run(E)
    p.check(first, want)
    again = p.run(E)
    for name, t in again.items():
        live = {"lse": p.live_q, "dk": p.live_k, "dv": p.live_k, "dtable": slice(None)}.get(name, p.live_q)
        assert torch.equal(t[live], first[name][live]), name
    p.check(p.run(E, hints=0), want)
