"""Which buffer a kept workspace hands out, without a GPU: buffers here are host memory."""
import gc
import weakref

import pytest
import torch

CPU = -1


@pytest.fixture
def ws():
    import paper_2512_01678_amd.gcn as G
    return G._Workspace()


def test_a_buffer_serves_its_stream(ws):
    a = ws.take(1000, CPU, 1, False)
    assert ws.take(1000, CPU, 1, False) is a and ws.take(10, CPU, 1, False) is a and ws.kept(0, CPU, 1, False) is a
    assert ws.kept(1001, CPU, 1, False) is None
    # another stream never sees it, though it is large enough
    assert ws.kept(0, CPU, 2, False) is None
    b = ws.take(10, CPU, 2, False)
    assert b is not a and b.untyped_storage().data_ptr() != a.untyped_storage().data_ptr()
    assert ws.kept(0, CPU, 1, False) is None and ws.take(10, CPU, 2, False) is b
    assert ws.kept(0, 0, 2, False) is None  # another device


def test_nothing_else_is_kept(ws):
    a = weakref.ref(ws.take(1000, CPU, 1, False))
    ws.take(2000, CPU, 1, False)
    gc.collect()
    assert a() is None


def test_what_a_graph_uses_stays(ws):
    a = ws.take(1000, CPU, 1, False)
    assert ws.take(500, CPU, 7, True) is a  # captured: what is there, whatever the stream
    assert ws.kept(500, CPU, 8, True) is a and len(ws.held) == 1
    assert ws.take(700, CPU, 1, False) is a  # and its own stream goes on with it
    at = weakref.ref(a)
    del a
    b = ws.take(5000, CPU, 1, False)  # replaced by a larger one
    gc.collect()
    assert at() is not None and b is not at()
    c = weakref.ref(ws.take(9000, CPU, 9, True))  # allocated under capture
    ws.take(20000, CPU, 1, False)
    del b
    gc.collect()
    assert c() is not None and len(ws.held) == 2


def test_refusals_of_the_calls_stream():
    """A stream of another device than the tensors' is refused before anything is looked at."""
    import paper_2512_01678_amd.gcn as G

    class Stream:
        device = torch.device("cuda", 1)

    with pytest.raises(ValueError):
        G._call(None, (), "call", None, 0, Stream())
