"""The largest sizes that the calls of the attention-based fusion take: on the host, before anything is enqueued."""
import ctypes as C

import pytest

from paper_2511_20564_b200 import binding as B

ARG = -2


def sizes(q_rows, k_rows, backward):
    """Answer of a size query of one head of eight bf16 values."""
    mat = lambda rows: C.byref(B.Mat(4096, rows, 8, 8, B.BF16))
    seqs, n, L = B.SequencesStruct(1, 4096, 4096, 0, 0, None), C.c_size_t(0), B.lib()
    q, k = mat(q_rows), mat(k_rows)
    if backward:
        return L.e2egrec_cross_attention_backward(q, q, k, k, q, None, C.byref(seqs), 1, 1, 1.0, q, k, k, None, None, C.byref(n), None)
    return L.e2egrec_cross_attention_forward(q, k, k, C.byref(seqs), 1, 1, 1.0, q, None, None, None, C.byref(n), None)


@pytest.mark.parametrize("backward", [False, True])
def test_rows_whose_steps_would_pass_32_bits_are_refused(backward):
    """The streaming kernels number a sequence's keys in 32 bits, and look up to 160 beyond the last (four warps' turns of 32, and a lane):
    with 2^31 - 1 keys those numbers were negative and passed for keys of the sequence."""
    most = (1 << 31) - (1 << 16)
    assert most + 4 * 32 + 32 < 1 << 31
    assert sizes(most, 1, backward) == 0 and sizes(1, most, backward) == 0
    for rows in (most + 1, (1 << 31) - 1):
        assert sizes(1, rows, backward) == ARG and sizes(rows, 1, backward) == ARG
