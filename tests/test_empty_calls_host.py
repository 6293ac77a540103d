"""Calls over no rows: two empty matrices have the same (null) address and may have any pitches.  Nothing is launched."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def G():
    import paper_2512_01678_amd.gcn as G
    return G


@pytest.mark.parametrize("at", [None, 4096])
def test_empty_matrices_are_not_in_place(G, at):
    L, big = G.raw_lib(), lambda: C.byref(G.sz(1 << 20))
    assert L.gcn_group_norm_fwd(0, 8, 2, 0, 64, -1, at, 8, None, None, 1e-5, 1, at, 12, None, None, 256, big(), None) == G.OK
    for dx in (None, at):
        assert L.gcn_group_norm_bwd(0, 8, 2, 0, 64, -1, at, 8, None, None, 1, None, None, at, 12, dx, 8, None, None, 256, big(),
                                    None) == G.OK
    for rows, cols in ((0, 8), (8, 0), (0, 0)):
        assert L.gcn_orthogonalize(rows, cols, at, 8, 5, at, 12, 256, big(), None) == G.OK


def test_with_rows_they_are(G):
    L, big = G.raw_lib(), lambda: C.byref(G.sz(1 << 40))
    assert L.gcn_group_norm_fwd(3, 8, 2, 1, None, -1, 4096, 8, None, None, 1e-5, 1, 4096, 12, 64, 64, 256, big(),
                                None) == G.E_INVALID
    assert L.gcn_group_norm_bwd(3, 8, 2, 1, None, -1, 4096, 8, None, None, 1, 64, 64, 8192, 12, 8192, 8, None, None, 256, big(),
                                None) == G.E_INVALID
    assert L.gcn_orthogonalize(3, 8, 4096, 8, 5, 4096, 12, 256, big(), None) == G.E_INVALID
