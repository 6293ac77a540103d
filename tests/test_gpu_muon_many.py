"""Optimiser steps over more matrices than one call of the library takes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    import paper_2512_01678_amd.gcn as G
    return G


def matrices(shapes, seed):
    rng = np.random.default_rng(seed)
    mk = lambda s: [torch.from_numpy((s * rng.standard_normal(x)).astype(np.float32)).cuda() for x in shapes]
    return mk(0.2), mk(1e-3), mk(1e-3)


SHAPES = [(100, 70), (70, 70), (30, 5), (0, 4), (128, 64), (7, 90)] * 6 + [(33, 200)]


@pytest.mark.parametrize("count", [16, 17, 32, 37])
def test_the_same_as_calls_of_sixteen(G, count):
    p, g, m = matrices(SHAPES[:count], 1)
    q, n = [t.clone() for t in p], [t.clone() for t in m]
    scales, ws = [0.5 + 0.1 * i for i in range(count)], G._Workspace()
    for _ in range(2):
        G.muon(p, g, m, weight_decay=0.1, scales=scales, ws=ws)
        for i in range(0, count, 16):
            s = slice(i, i + 16)
            G.muon(q[s], g[s], n[s], weight_decay=0.1, scales=scales[s])
    assert all(torch.equal(a, b) for a, b in zip(p + m, q + n))


def test_captured(G):
    p, g, m = matrices(SHAPES, 2)
    q, n = [t.clone() for t in p], [t.clone() for t in m]
    keep = G._Workspace()
    warm = [t.clone() for t in p], [t.clone() for t in m]
    G.muon(warm[0], g, warm[1], ws=keep)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.muon(p, g, m, ws=keep)
    for rep in range(3):
        graph.replay()
        G.muon(q, g, n)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(p + m, q + n)), rep


def test_refused_as_a_whole(G):
    """What only a later call of the library would refuse leaves the matrices of the first alone."""
    p, g, m = matrices(SHAPES, 3)
    was = [t.clone() for t in p + m]
    long = torch.zeros((1 << 24) + 1, 1, device="cuda")  # a side that the library does not take
    swap = lambda ts, i, t: ts[:i] + [t] + ts[i + 1:]
    for args in ((swap(p, 36, p[2]), swap(g, 36, g[2]), swap(m, 36, torch.zeros_like(m[2]))),  # a parameter twice
                 (p, g, swap(m, 24, m[0])), (p, swap(g, 24, m[0]), m), (p, swap(g, 24, p[0]), m),
                 (p + [long], g + [torch.zeros_like(long)], m + [torch.zeros_like(long)])):
        with pytest.raises((ValueError, G.GcnError)):
            G.muon(*args)
    with pytest.raises(G.GcnError):
        G.muon(p, g, m, steps=65)
    with pytest.raises(G.GcnError):
        G.muon(p, g, m, scales=[1.0] * 36 + [float("nan")])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(p + m, was))
    G.muon(p, [g[2] if t.shape == g[2].shape else t for t in g], m)  # a gradient may be shared
