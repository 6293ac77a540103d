"""Optimiser steps over matrices that the one-workgroup form takes one by one, but not together: up to 32 x 1,536
beside up to 64 x 768.  Its limits are those of the largest shorter and the largest longer side of the call."""
import ctypes as C

import numpy as np
import pytest
import torch

import muon_ref as ref

U = 2.0 ** -24


@pytest.fixture(scope="module")
def G():
    import paper_2512_01678_amd.gcn as G
    return G


def need(G, shapes):
    arr, nb = (G.gcn_muon_tensor * len(shapes))(), G.sz(1)
    for i, (r, c) in enumerate(shapes):
        arr[i] = G.gcn_muon_tensor(256, 512, 1024, r, c, 1.0)
    assert G.raw_lib().gcn_muon(arr, len(shapes), 5, 0.02, 0.95, 1, 0.0, None, C.byref(nb), None) == G.OK
    return nb.value


MIXED = [[(20, 1500), (60, 100)], [(1536, 32), (768, 64), (3, 2), (0, 9)], [(33, 768), (1000, 7), (64, 64), (32, 1536)]]


@pytest.mark.parametrize("shapes", MIXED)
def test_workspace_of_small_matrices(G, shapes):
    for s in shapes:
        assert need(G, [s]) == 0
    assert need(G, shapes) > 0
    assert need(G, [s for s in shapes if min(s) <= 32]) == 0 and need(G, [s for s in shapes if max(s) <= 768]) == 0
    for s in ((33, 769), (65, 65), (32, 1537), (769, 64)):
        assert need(G, [s]) > 0


@pytest.mark.gpu
@pytest.mark.parametrize("shapes", MIXED)
def test_steps(G, shapes):
    rng = np.random.default_rng(1)
    mk = lambda s: [(s * rng.standard_normal(x)).astype(np.float32) for x in shapes]
    p, g, m = mk(0.2), mk(1e-3), mk(1e-3)
    dev = lambda ts: [torch.from_numpy(t).cuda() for t in ts]
    P, D, M = dev(p), dev(g), dev(m)
    lr, mu, wd, scales = 0.02, 0.9, 0.1, [0.5 + 0.25 * i for i in range(len(shapes))]
    G.muon(P, D, M, lr=lr, momentum=mu, weight_decay=wd, scales=scales)
    for i, s in enumerate(shapes):
        if not p[i].size:
            continue
        want_p, want_m, u = ref.step(p[i].astype(np.float64), g[i].astype(np.float64), m[i].astype(np.float64), lr, mu,
                                     True, wd, scales[i])
        want = ref.newton_schulz(u)
        # of the orthogonalised update: its own distance, and that of u, which carries up to 4 roundings of terms no
        # larger than |m| + |g|, amplified like the products' own roundings; three roundings of p and of m
        noise = 4 * U * (np.linalg.norm(g[i]) + np.linalg.norm(m[i])) / np.linalg.norm(u) * 3.4445 ** 5
        tol = lr * scales[i] * np.linalg.norm(want) * (ref.allowed(u.astype(np.float32), want) + noise) \
            + 3 * U * np.linalg.norm(p[i])
        assert np.linalg.norm(P[i].cpu().numpy() - want_p) <= tol, s
        assert np.abs(M[i].cpu().numpy() - want_m).max() <= 3 * U * (np.abs(m[i]).max() + np.abs(g[i]).max()), s
