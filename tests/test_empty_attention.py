"""Attention of nothing: calls that enqueue nothing ask nothing of a device, so they succeed where there is none."""
import ctypes as C

import pytest

from paper_2511_20564_b200 import binding as B

P = C.c_void_p(4096)


@pytest.mark.parametrize("n_seq,rows", [(0, 0), (0, 4), (2, 0)])
def test_empty_calls_enqueue_nothing(n_seq, rows):
    L, s, n = B.lib(), B.SequencesStruct(n_seq, 4096, 4096, 0, 0, None), C.c_size_t(1 << 40)
    m = lambda dim=256: C.byref(B.Mat(4096, rows, dim, dim, B.BF16))
    bias = C.byref(B.RelativeBiasStruct(8, 4096, 4096, None, None))
    before = L.e2egrec_launch_count()
    assert L.e2egrec_cross_attention_forward(m(), m(128), m(128), C.byref(s), 4, 2, 1.0, m(), None, None, P, C.byref(n), None) == 0
    assert L.e2egrec_biased_attention_forward(m(), m(128), m(128), C.byref(s), bias, 4, 2, 1.0, m(), None, None, P, C.byref(n), None) == 0
    assert L.e2egrec_cross_attention_backward(m(), m(), m(128), m(128), m(), P, C.byref(s), 4, 2, 1.0, m(), m(128), m(128), None, P, C.byref(n), None) == 0
    assert L.e2egrec_biased_attention_backward(m(), m(), m(128), m(128), m(), P, C.byref(s), bias, 4, 2, 1.0, m(), m(128), m(128), None, None, P,
                                               C.byref(n), None) == 0
    assert L.e2egrec_launch_count() == before
