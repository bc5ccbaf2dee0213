"""What attention with a bias refuses, and its size queries: all on the host, before anything is enqueued."""
import ctypes as C

import pytest
import torch

import paper_2511_20564_b200 as E
from paper_2511_20564_b200 import binding as B

NULL, ARG, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4, -5, -6
P = C.c_void_p(4096)


def mat(rows=4, dim=128, ld=None, dtype=B.BF16, data=4096):
    return C.byref(B.Mat(data, rows, dim, dim if ld is None else ld, dtype))


def bias(n=8, edges=4096, table=4096, pos_q=4096, pos_k=4096):
    return C.byref(B.RelativeBiasStruct(n, edges, table, pos_q, pos_k))


def forward(b="bias", q=None, k=None, v=None, out=None, n_seq=2, heads=4, kv=2, scale=1.0, ws=P, n=None):
    s, n = B.SequencesStruct(n_seq, 4096, 4096, 0, 0, None), C.c_size_t(1 << 40) if n is None else n
    return B.lib().e2egrec_biased_attention_forward(q or mat(dim=256), k or mat(), v or mat(), C.byref(s), bias() if b == "bias" else b, heads, kv, scale,
                                                    out or mat(dim=256), None, None, ws, C.byref(n), None)


def backward(b="bias", dout=None, dk=None, dtable=P, lse=P, ws=P, n=None):
    s, n = B.SequencesStruct(2, 4096, 4096, 0, 0, None), C.c_size_t(1 << 40) if n is None else n
    return B.lib().e2egrec_biased_attention_backward(dout or mat(dim=256), mat(dim=256), mat(), mat(), mat(dim=256), lse, C.byref(s),
                                                     bias() if b == "bias" else b, 4, 2, 1.0, mat(dim=256), dk or mat(), mat(), dtable, None, ws,
                                                     C.byref(n), None)


def test_bias_refusals():
    for call in (forward, backward):
        assert call(b=None) == NULL and call(b=bias(table=None)) == NULL and call(b=bias(edges=None)) == NULL
        assert call(b=bias(n=0)) == ARG and call(b=bias(n=-3)) == ARG and call(b=bias(n=129)) == UNSUPPORTED
        for name in ("edges", "table", "pos_q", "pos_k"):
            assert call(b=bias(**{name: 4098})) == ALIGN, name
        n = C.c_size_t(0)
        assert call(ws=None, n=n) == 0 and n.value > 0 and call(n=C.c_size_t(n.value - 1)) == WORKSPACE
        assert call(b=bias(table=None, edges=None), ws=None, n=n) == 0              # a size query has no pointers
        assert call(ws=C.c_void_p(4100)) == ALIGN
    wide = dict(q=mat(dim=8 * 1024), out=mat(dim=8 * 1024), k=mat(dim=8), v=mat(dim=8), heads=1024, kv=1)
    assert forward(b=bias(n=65), **wide) == UNSUPPORTED
    # what the call without a bias refuses
    assert forward(scale=0.0) == ARG and forward(heads=3) == ARG and forward(v=mat(rows=3)) == ARG and forward(q=mat(dim=256, dtype=5)) == DTYPE
    assert forward(out=mat(dim=256, ld=260)) == ALIGN and forward(n_seq=-1) == ARG
    assert backward(dout=mat(rows=3, dim=256)) == ARG and backward(dk=mat(data=4100)) == ALIGN and backward(lse=None) == NULL
    assert backward(dtable=C.c_void_p(4097)) == ALIGN


def test_the_binding_refuses_what_the_library_cannot_see():
    table, edges = torch.zeros(4, 2), torch.zeros(3, dtype=torch.int32)
    x, ptr = torch.zeros(4, 64), torch.tensor([0, 2, 4])
    for bad in (lambda: E.RelativeBias(table.double(), edges), lambda: E.RelativeBias(table, edges.long()), lambda: E.RelativeBias(table, edges[:2]),
                lambda: E.RelativeBias(table[0], edges), lambda: E.RelativeBias(table.T, edges[:1]),
                lambda: E.biased_attention_forward(x, x, x, E.Sequences(ptr, ptr), E.RelativeBias(table, edges), 2, 2, 1.0)):
        with pytest.raises(E.E2EGrecError):
            bad()
