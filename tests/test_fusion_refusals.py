"""What the calls of the attention-based fusion refuse, and their size queries: all on the host, before anything is enqueued."""
import ctypes as C

import pytest
import torch

import paper_2511_20564_b200 as E
from paper_2511_20564_b200 import binding as B

NULL, ARG, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4, -5, -6
P = C.c_void_p(4096)


def mat(rows=4, dim=128, ld=None, dtype=B.BF16, data=4096):
    return C.byref(B.Mat(data, rows, dim, dim if ld is None else ld, dtype))


def rotary(x=None, heads=2, freqs=P, rot=64, pos=P, scale=1.0, flags=0, y=None):
    return B.lib().e2egrec_rotary(x or mat(), heads, freqs, rot, pos, scale, flags, y or mat(), None)


def norm(q=None, k=None, heads=2, kv=1, eps=1e-6, rot=64, freqs=P, scale=1.0, flags=0, qn=None, kn=None):
    return B.lib().e2egrec_qk_norm_rotary_forward(q or mat(), k, heads, kv, None, None, eps, freqs, rot, None, None, scale, flags,
                                                  qn or mat(), kn, None)


def test_rotary_refusals():
    L = B.lib()
    assert L.e2egrec_rotary(None, 2, P, 64, P, 1.0, 0, mat(), None) == NULL
    assert L.e2egrec_rotary(mat(), 2, P, 64, P, 1.0, 0, None, None) == NULL
    assert rotary(mat(data=None)) == NULL and rotary(freqs=None) == NULL
    for bad in (dict(heads=0), dict(heads=3), dict(rot=66), dict(rot=63), dict(rot=-2), dict(scale=0.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(flags=4), dict(x=mat(rows=-1)), dict(x=mat(rows=1 << 31)), dict(y=mat(rows=3)),
                dict(y=mat(dim=64)), dict(x=mat(ld=120))):
        assert rotary(**bad) == ARG, bad
    assert rotary(x=mat(dtype=7)) == DTYPE and rotary(y=mat(dtype=B.F32)) == DTYPE
    for bad in (dict(x=mat(ld=132)), dict(x=mat(data=4104)), dict(y=mat(data=4098)), dict(x=mat(dim=72), y=mat(dim=72), rot=4)):
        assert rotary(**bad) == ALIGN, bad
    assert rotary(x=mat(dim=1024), y=mat(dim=1024), rot=64) == UNSUPPORTED            # heads of 512
    assert rotary(x=mat(rows=0), y=mat(rows=0)) == 0                                  # nothing to do
    f = L.e2egrec_rotary_frequencies
    for bad in ((0, 1e4, 1.0, 0.0, 1.0, 2.0), (7, 1e4, 1.0, 0.0, 1.0, 2.0), (8, 0.0, 1.0, 0.0, 1.0, 2.0), (8, 1e4, 0.5, 0.0, 1.0, 2.0),
                (8, 1e4, 1.0, 0.0, 2.0, 2.0), (8, 1e4, 1.0, -1.0, 1.0, 2.0)):
        assert f(*bad, P, None) == ARG, bad
    assert f(512, 1e4, 1.0, 0.0, 1.0, 2.0, P, None) == UNSUPPORTED and f(8, 1e4, 1.0, 0.0, 1.0, 2.0, None, None) == NULL


def test_qk_norm_refusals():
    assert norm(heads=0) == ARG and norm(heads=3) == ARG and norm(eps=-1.0) == ARG and norm(eps=float("nan")) == ARG
    assert norm(flags=2) == ARG and norm(rot=130) == ARG and norm(freqs=None) == NULL
    assert norm(k=mat(dim=64), kn=None) == NULL and norm(k=mat(dim=64), kn=mat(dim=128)) == ARG and norm(k=mat(dim=128), kn=mat(dim=128)) == ARG
    assert norm(k=mat(dim=64, dtype=B.F32), kn=mat(dim=64)) == DTYPE and norm(k=mat(dim=64), kv=0, kn=mat(dim=64)) == ARG
    assert norm(k=mat(dim=64, data=4100), kn=mat(dim=64)) == ALIGN and norm(qn=mat(rows=2)) == ARG
    L, n = B.lib(), C.c_size_t(0)

    def back(ws, n, dqn=None, dq=None, wsb=True):
        return L.e2egrec_qk_norm_rotary_backward(dqn or mat(), None, mat(), None, 2, 1, None, None, 1e-6, P, 64, None, None, 1.0, 0,
                                                 dq or mat(), None, None, None, ws, C.byref(n) if wsb else None, None)

    assert back(None, n) == 0 and n.value > 0
    assert back(P, C.c_size_t(8)) == WORKSPACE and back(C.c_void_p(4097), n) == ALIGN and back(P, n, wsb=False) == NULL
    assert back(P, n, dqn=mat(rows=3)) == ARG and back(P, n, dq=mat(data=None)) == NULL and back(P, n, dq=mat(dtype=B.F32)) == DTYPE


def attend(q=None, k=None, v=None, out=None, n_seq=2, qp=4096, kp=4096, mq=0, mk=0, heads=4, kv=2, scale=1.0, ws=P, n=None, seqs=True):
    s = B.SequencesStruct(n_seq, qp, kp, mq, mk, None)
    n = C.c_size_t(1 << 40) if n is None else n
    return B.lib().e2egrec_cross_attention_forward(q or mat(dim=256), k or mat(), v or mat(), C.byref(s) if seqs else None, heads, kv, scale,
                                                   out or mat(dim=256), None, None, ws, C.byref(n), None)


def test_attention_refusals():
    for bad in (dict(heads=0), dict(kv=0), dict(kv=3), dict(heads=2, kv=4), dict(heads=3, kv=3), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("nan")), dict(n_seq=-1), dict(mq=-1), dict(mk=-1), dict(q=mat(rows=-1, dim=256)),
                dict(k=mat(rows=1 << 31)), dict(k=mat(dim=256)), dict(v=mat(rows=3)), dict(v=mat(dim=64)), dict(out=mat(rows=3, dim=256)),
                dict(out=mat(dim=128)), dict(k=mat(ld=64))):
        assert attend(**bad) == ARG, bad
    for bad in (dict(seqs=False), dict(qp=None), dict(kp=None), dict(q=mat(dim=256, data=None)), dict(v=mat(data=None))):
        assert attend(**bad) == NULL, bad
    for bad in (dict(q=mat(dim=256, dtype=5)), dict(k=mat(dtype=B.F32)), dict(v=mat(dtype=B.F32)), dict(out=mat(dim=256, dtype=B.F32))):
        assert attend(**bad) == DTYPE, bad
    for bad in (dict(q=mat(dim=256, data=4104)), dict(k=mat(ld=132)), dict(out=mat(dim=256, ld=260)), dict(ws=C.c_void_p(4100)),
                dict(q=mat(dim=16), out=mat(dim=16), k=mat(dim=8), v=mat(dim=8))):
        assert attend(**bad) == ALIGN, bad
    assert attend(q=mat(dim=2048), k=mat(dim=1024), v=mat(dim=1024), out=mat(dim=2048)) == UNSUPPORTED
    n = C.c_size_t(0)
    assert attend(ws=None, n=n) == 0 and n.value > 0
    assert attend(n=C.c_size_t(n.value - 1)) == WORKSPACE
    assert attend(n_seq=0, qp=None, kp=None) == 0                   # nothing to do
    s, L = B.SequencesStruct(2, 4096, 4096, 0, 0, None), B.lib()

    def back(dout=None, out=None, lse=P, dq=None, dk=None, dv=None, ws=P, n=None, seqs=s):
        n = C.c_size_t(1 << 40) if n is None else n
        return L.e2egrec_cross_attention_backward(dout or mat(dim=256), mat(dim=256), mat(), mat(), out or mat(dim=256), lse, C.byref(seqs), 4, 2,
                                                  1.0, dq or mat(dim=256), dk or mat(), dv or mat(), None, ws, C.byref(n), None)

    assert back(ws=None, n=n) == 0 and n.value > 0 and back(n=C.c_size_t(n.value - 1)) == WORKSPACE
    assert back(dout=mat(rows=3, dim=256)) == ARG and back(dk=mat(rows=3)) == ARG and back(dv=mat(dim=64)) == ARG
    assert back(lse=None) == NULL and back(dq=mat(dim=256, data=None)) == NULL and back(out=mat(dim=256, dtype=B.F32)) == DTYPE
    assert back(dk=mat(data=4100)) == ALIGN and back(seqs=B.SequencesStruct(2, None, 4096, 0, 0, None)) == NULL


def test_the_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(4, 64)
    with pytest.raises(E.E2EGrecError):
        E.rotary(x, 2, None)
    ptr = torch.tensor([0, 2, 4])
    for bad in (lambda: E.Sequences(ptr.int(), ptr), lambda: E.Sequences(ptr, ptr[:2]), lambda: E.Sequences(ptr, ptr, k_mask=torch.zeros(4)),
                lambda: E.cross_attention_forward(x, x, x, E.Sequences(ptr, ptr), 2, 2, 1.0),
                lambda: E.qk_norm_rotary_forward(x, None, 2, 1)):
        with pytest.raises(E.E2EGrecError):
            bad()
