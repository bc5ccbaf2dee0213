"""What dropout and layer norm refuse, and their size queries: all on the host, before anything is enqueued."""
import ctypes as C

import pytest
import torch

import paper_2511_20564_b200 as E
from paper_2511_20564_b200 import binding as B

NULL, ARG, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4, -5, -6
P = C.c_void_p(4096)


def mat(rows=4, dim=64, ld=None, dtype=B.BF16, data=4096):
    return C.byref(B.Mat(data, rows, dim, dim if ld is None else ld, dtype))


def plan(p=0.1, place=0, step_dev=None):
    return C.byref(B.DropoutStruct(p, 1, place, 0, step_dev))


BAD_PLANS = [(plan(-0.1), ARG), (plan(1.0), ARG), (plan(float("nan")), ARG), (plan(place=1 << 31), ARG), (plan(step_dev=4097), ALIGN)]
# every matrix beside X: what is wrong with it
BAD_MATS = [(dict(rows=3), ARG), (dict(dim=128), ARG), (dict(ld=56), ARG), (dict(dtype=B.F32), DTYPE), (dict(dtype=9), DTYPE), (dict(data=None), NULL),
            (dict(data=4104), ALIGN), (dict(ld=68), ALIGN)]
BAD_X = [(dict(rows=-1), ARG), (dict(rows=1 << 31), ARG), (dict(dim=0, ld=8), ARG), (dict(dim=60), ALIGN), (dict(dtype=9), DTYPE), (dict(data=None), NULL)]


def test_dropout_refusals():
    f = B.lib().e2egrec_dropout_apply
    for p, code in BAD_PLANS:
        assert f(mat(), None, p, mat(), None) == code
    for kw, code in BAD_MATS:
        assert f(mat(), None, plan(), mat(**kw), None) == code, kw
        assert f(mat(), mat(**kw), plan(), mat(), None) == code, kw
    for kw, code in BAD_X:
        assert f(mat(**kw), None, plan(), mat(**kw), None) == code, kw
    assert f(None, None, plan(), mat(), None) == NULL and f(mat(), None, plan(), None, None) == NULL
    assert f(mat(rows=0, data=None), None, plan(), mat(rows=0, data=None), None) == 0          # nothing to do


def forward(x=None, r=None, p=None, gain=P, shift=P, eps=1e-5, y=None, z=None, stats=P):
    return B.lib().e2egrec_layer_norm_forward(x or mat(), r, p, gain, shift, eps, y or mat(), z, stats, None)


def backward(dy=None, dz=None, x=None, r=None, p=None, gain=P, stats=P, dx=None, dr=None, ws=P, n=None, sized=True):
    n = C.c_size_t(1 << 40) if n is None else n
    return B.lib().e2egrec_layer_norm_backward(dy or mat(), dz, x or mat(), r, p, gain, stats, dx or mat(), dr, P, P, ws, C.byref(n) if sized else None, None)


def test_layer_norm_refusals():
    for p, code in BAD_PLANS:
        assert forward(p=p) == code and backward(p=p) == code
    for kw, code in BAD_MATS:
        for name in ("r", "y", "z"):
            assert forward(**{name: mat(**kw)}) == code, (name, kw)
        for name in ("dy", "dz", "r", "dx", "dr"):
            assert backward(**{name: mat(**kw)}) == code, (name, kw)
    for kw, code in BAD_X:
        assert forward(x=mat(**kw), y=mat(**kw)) == code and backward(x=mat(**kw), dy=mat(**kw), dx=mat(**kw)) == code, kw
    for eps in (0.0, -1e-5, float("nan")):
        assert forward(eps=eps) == ARG
    odd, wide = C.c_void_p(4100), dict(dim=8200)
    assert forward(gain=odd) == ALIGN and forward(shift=odd) == ALIGN and forward(stats=odd) == ALIGN
    assert backward(gain=odd) == ALIGN and backward(stats=odd) == ALIGN and backward(ws=C.c_void_p(4097)) == ALIGN
    assert forward(x=mat(**wide), y=mat(**wide)) == UNSUPPORTED and backward(x=mat(**wide)) == UNSUPPORTED
    assert backward(stats=None) == NULL and backward(sized=False) == NULL
    n = C.c_size_t(0)
    assert backward(ws=None, n=n) == 0 and n.value > 0
    assert backward(n=C.c_size_t(n.value - 1)) == WORKSPACE
    assert forward(x=mat(rows=0), y=mat(rows=0)) == 0


def test_the_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(4, 64)
    for bad in (lambda: E.Dropout(1.0, 1), lambda: E.Dropout(-0.5, 1), lambda: E.Dropout(0.1, 1, place=-1), lambda: E.Dropout(0.1, 1, place=1 << 31),
                lambda: E.Dropout(0.1, 1, step_dev=torch.zeros(2, dtype=torch.int32)), lambda: E.Dropout(0.1, 1, step_dev=torch.zeros(1)),
                lambda: E.dropout(x, None), lambda: E.layer_norm_forward(x), lambda: E.layer_norm_backward(x, x, None)):
        with pytest.raises(E.E2EGrecError):
            bad()


def test_two_results_in_one_place_are_refused():
    other = mat(data=8192)
    assert forward(y=mat(), z=mat()) == ARG and backward(dx=mat(), dr=mat()) == ARG
    assert forward(x=mat(rows=0), y=mat(rows=0), z=mat(rows=0)) == 0
    n = C.c_size_t(1 << 40)
    for k in (0, 1):
        gains = [P, P]
        gains[k] = C.c_void_p(4097)
        assert B.lib().e2egrec_layer_norm_backward(mat(), None, mat(), None, None, P, P, mat(), other, *gains, P, C.byref(n), None) == ALIGN
