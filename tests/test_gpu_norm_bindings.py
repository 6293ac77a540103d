"""What the binding's calls take: statistics of any layout in the backward pass, and a workspace that goes from
stream to stream and into graphs."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    import paper_2512_01678_amd.gcn as G
    return G


def batch(n, c, k, seed):
    rng = np.random.default_rng(seed)
    ptr = [0, *np.sort(rng.integers(0, n + 1, k - 1)).tolist(), n]
    dev = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()
    return dev(n, c), dev(n, c), dev(c), dev(c), torch.tensor(ptr, device="cuda")


def layouts(v):
    """The same values with rows or columns apart, and as a copy with none."""
    k, g = v.shape
    wide, tall = torch.full((k + 2, g + 3), 9.0, device="cuda"), torch.full((g + 1, k + 5), 9.0, device="cuda")
    wide[1:k + 1, 2:g + 2] = v
    tall[:g, 1:k + 1] = v.T
    return dict(dense=v.clone(), turned=v.T.clone(memory_format=torch.contiguous_format).T, slice=wide[1:k + 1, 2:g + 2], turned_slice=tall[:g, 1:k + 1].T)


@pytest.mark.parametrize("k,groups", [(1, 1), (1, 4), (5, 1), (5, 4), (300, 8)])
def test_backward_takes_statistics_of_any_layout(G, k, groups):
    x, dy, ga, be, seg = batch(900, 16, k, 1)
    kw = dict(seg_ptr=seg, max_seg=900, act=G.ACT_SILU)
    mean, rstd = torch.empty(k, groups, device="cuda"), torch.empty(k, groups, device="cuda")
    G.group_norm(x, groups, ga, be, torch.empty_like(x), mean, rstd, **kw)

    def run(mean, rstd, stream=None):
        out = torch.zeros_like(x), torch.zeros_like(ga), torch.zeros_like(be)
        torch.cuda.synchronize()
        G.group_norm_bwd(x, dy, mean, rstd, groups, ga, be, *out, stream=stream, **kw)
        torch.cuda.synchronize()
        return out

    want = run(mean, rstd)
    means, rstds = layouts(mean), layouts(rstd)
    for a in means:
        for b in rstds:
            for stream in (None, torch.cuda.Stream()):
                for got, w in zip(run(means[a], rstds[b], stream), want):
                    assert torch.equal(got, w), (a, b)
    # captured: the copy is part of the graph, and takes the values of the time of the replay
    out, turned = [torch.zeros_like(w) for w in want], [means["turned"], rstds["turned"]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.group_norm_bwd(x, dy, *turned, groups, ga, be, *out, **kw)
    for rep in range(3):
        for t, v in zip(turned, (mean, rstd)):
            t.copy_(v * (1 + rep))
        expect = run(mean * (1 + rep), rstd * (1 + rep))
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip(out, expect):
            assert torch.equal(got, w), rep


def test_statistics_with_gaps_or_overlaps_are_refused(G):
    x, dy, ga, be, seg = batch(40, 8, 3, 2)
    z = lambda *s: torch.zeros(*s, device="cuda")
    ok = z(3, 2)
    for bad in (z(3, 4)[:, ::2], z(1, 2).expand(3, 2), z(3, 1).expand(3, 2), z(2, 3), z(4, 2), z(3, 2).double(),
                z(3, 2).cpu(), z(6), z(3, 2, 1)):
        for args in ((bad, ok), (ok, bad)):
            with pytest.raises(ValueError):
                G.group_norm_bwd(x, dy, *args, 2, ga, be, torch.zeros_like(x), seg_ptr=seg)
    # what is written has to be dense; a row of a wider buffer is
    for bad in (z(2, 3).T, z(3, 4)[:, :2]):
        for args in ((bad, ok), (ok, bad)):
            with pytest.raises(ValueError):
                G.group_norm(x, 2, ga, be, torch.zeros_like(x), *args, seg_ptr=seg)
    mean, rstd = z(5, 7)[2:3, 1:3], z(5, 7)[2:3, 1:3]
    dense = z(1, 2), z(1, 2)
    y, w = torch.zeros_like(x), torch.zeros_like(x)
    G.group_norm(x, 2, ga, be, y, mean, rstd)
    G.group_norm(x, 2, ga, be, w, *dense)
    assert torch.equal(y, w) and torch.equal(mean, dense[0]) and torch.equal(rstd, dense[1])


def test_a_workspace_that_goes_from_stream_to_stream(G):
    """Calls on two streams in turn, growing, with other work of both streams beside them: every result as alone."""
    cases = [(3000 + 40000 * i, 64, 1 + 3 * i) for i in range(4)]
    data = [batch(n, c, k, i) for i, (n, c, k) in enumerate(cases)]

    def buffers(n, c, k):
        z = lambda *s: torch.zeros(*s, device="cuda")
        return z(n, c), z(k, 8), z(k, 8), z(n, c), z(c), z(c)

    def run(i, o, ws, stream=None):
        x, dy, ga, be, seg = data[i]
        kw = dict(seg_ptr=seg, act=G.ACT_SILU, ws=ws, stream=stream)
        G.group_norm(x, 8, ga, be, o[0], o[1], o[2], **kw)
        G.group_norm_bwd(x, dy, o[1], o[2], 8, ga, be, o[3], o[4], o[5], **kw)

    want = [buffers(*c) for c in cases]
    for i in range(4):
        run(i, want[i], None)
    work = torch.ones(1 << 26, device="cuda")
    streams = [None, torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(3):
        got, ws = [buffers(*c) for c in cases], G._Workspace()
        torch.cuda.synchronize()
        for i in range(4):
            s = streams[(turn + i) % 3]
            with torch.cuda.stream(s):
                for _ in range(5):
                    work.mul_(1.0) if s is None else torch.ones(1 << 24, device="cuda")
            run(i, got[i], ws, s)
            junk = [torch.full((v,), float("nan"), device="cuda") for v in (1 << 12, 1 << 16, 1 << 20) for _ in range(20)]
            assert junk
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for a, b in zip(g, w):
                assert torch.equal(a, b), turn


def test_a_graph_keeps_its_scratch_when_the_workspace_grows(G):
    x, dy, ga, be, seg = batch(50000, 64, 9, 1)
    z = lambda *s: torch.zeros(*s, device="cuda")
    y, mean, rstd, ws = z(50000, 64), z(9, 8), z(9, 8), G._Workspace()
    kw = dict(seg_ptr=seg, act=G.ACT_SILU)
    G.group_norm(x, 8, ga, be, y, mean, rstd, ws=ws, **kw)
    want, small = y.clone(), ws.buf
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.group_norm(x, 8, ga, be, y, mean, rstd, ws=ws, **kw)
    big = torch.randn(700, 700, device="cuda")
    G.orthogonalize(big, torch.empty_like(big), ws=ws)
    assert ws.buf is not small and any(b is small for b in ws.held)
    at = small.data_ptr()
    del small
    for rep in range(3):
        junk = [torch.full((v,), float("nan"), device="cuda") for v in (1 << 12, 1 << 16, 1 << 20) for _ in range(20)]
        assert all(t.data_ptr() != at for t in junk)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), rep


def test_the_other_calls_on_another_stream(G):
    """Products and column sums, with a workspace that goes from stream to stream and with none: the scratch is the
    stream's own, and what the current stream allocates meanwhile is other memory."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    a, b = torch.randn(20000, 64, device="cuda", generator=gen), torch.randn(20000, 48, device="cuda", generator=gen)
    want, sums = torch.zeros(64, 48, device="cuda"), torch.zeros(64, device="cuda")
    G.gemm(G.OP_TN, a, b, want)
    G.column_sums(a, sums)
    side, work = torch.cuda.Stream(), torch.ones(1 << 26, device="cuda")
    for ws in (None, G._Workspace()):
        for stream in (None, side, None, torch.cuda.default_stream(), side):
            got, got_sums = torch.zeros_like(want), torch.zeros_like(sums)
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                for _ in range(5):
                    work.mul_(1.0)
            G.gemm(G.OP_TN, a, b, got, ws=ws, stream=stream)
            G.column_sums(a, got_sums, stream=stream)
            junk = [torch.full((v,), float("nan"), device="cuda") for v in (1 << 12, 1 << 16, 1 << 20) for _ in range(20)]
            assert junk
            if ws is not None:
                assert ws.stream == (side if stream is side else torch.cuda.default_stream()).cuda_stream
            torch.cuda.synchronize()
            assert torch.equal(got, want) and torch.equal(got_sums, sums)
    # the call on the default stream, while another is current
    with torch.cuda.stream(side):
        got = torch.zeros_like(want)
        torch.cuda.synchronize()
        G.gemm(G.OP_TN, a, b, got, ws=ws, stream=torch.cuda.default_stream())
        torch.cuda.synchronize()
        assert torch.equal(got, want) and ws.stream == torch.cuda.default_stream().cuda_stream
