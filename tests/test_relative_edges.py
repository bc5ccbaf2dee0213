"""Sizes that e2egrec_relative_edges refuses, those beyond 32 bits among them, without an array that they would need."""
import pytest

import paper_2511_20564_b200 as E
from paper_2511_20564_b200 import binding as B

NULL, ARG, UNSUPPORTED = -1, -2, -6
TOP = 2 ** 31 - 1


@pytest.mark.parametrize("both,most", [(0, 128), (1, 64)])
def test_the_library_refuses_more_buckets_than_there_may_be(both, most):
    edges = B.lib().e2egrec_relative_edges
    for n in (most + 1, 2 ** 16, 2 ** 30, 2 ** 30 + 1, 2 ** 30 + 70, TOP):
        assert edges(n, 100, both, None) == UNSUPPORTED, n
    assert edges(most, 100, both, None) == NULL and edges(1, 100, both, None) == 0
    assert edges(0, 100, both, None) == ARG and edges(-TOP, 100, both, None) == ARG


@pytest.mark.parametrize("both", [False, True])
def test_the_binding_passes_no_number_on_that_does_not_fit(both):
    for n in (129, TOP, 2 ** 32 + 4, 2 ** 64 + 4, 0, -5, -(2 ** 32) + 4):
        with pytest.raises(E.E2EGrecError):
            E.relative_edges(n, 100, both, device="cpu")
    for far in (0, 2 ** 30 + 1, 2 ** 64 + 5, -(2 ** 64) + 5):
        with pytest.raises(E.E2EGrecError):
            E.relative_edges(8, far, both, device="cpu")
    most = 64 if both else 128
    edges = E.relative_edges(most, 2 ** 30, both, device="cpu").tolist()
    assert len(edges) == (2 * most - 2 if both else most - 1) and all(a < b for a, b in zip(edges, edges[1:]))
    assert E.relative_edges(1, 1, both, device="cpu").numel() == 0
