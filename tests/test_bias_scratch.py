"""Scratch of the backward pass of attention with a bias: rows of the table's gradient only where that is wanted."""
import ctypes as C

import pytest

from paper_2511_20564_b200 import binding as B

P = C.c_void_p(4096)
WORKSPACE = -5


def backward(rows, n_seq, heads, kv, hd, dtype, buckets, dtable, ws, n, max_q=0, bias=True):
    q, k = (lambda h=h: C.byref(B.Mat(4096, rows, h * hd, h * hd, dtype)) for h in (heads, kv))
    s, b = B.SequencesStruct(n_seq, 4096, 4096, max_q, max_q, None), B.RelativeBiasStruct(buckets, 4096, 4096, None, None)
    if not bias:
        return B.lib().e2egrec_cross_attention_backward(q(), q(), k(), k(), q(), P, C.byref(s), heads, kv, 1.0, q(), k(), k(), None, ws, C.byref(n), None)
    return B.lib().e2egrec_biased_attention_backward(q(), q(), k(), k(), q(), P, C.byref(s), C.byref(b), heads, kv, 1.0, q(), k(), k(), dtable, None, ws,
                                                     C.byref(n), None)


@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
@pytest.mark.parametrize("rows,n_seq,max_q", [(100_000, 100_000, 1), (4096, 2, 2048), (3000, 50, 0)])
def test_a_call_without_the_tables_gradient_needs_no_rows_of_it(rows, n_seq, max_q, dtype):
    args = (rows, n_seq, 64, 64, 32, dtype, 16)
    asked, full, less, plain = (C.c_size_t(0) for _ in range(4))
    assert backward(*args, None, None, asked, max_q) == 0                       # a size query: enough for either call
    assert backward(*args, P, P, full, max_q) == WORKSPACE and full.value == asked.value
    assert backward(*args, None, P, less, max_q) == WORKSPACE and 256 <= less.value < full.value
    assert full.value - less.value >= 64 * 16 * 4
    assert backward(*args, None, None, plain, max_q, bias=False) == 0 and plain.value >= 256
