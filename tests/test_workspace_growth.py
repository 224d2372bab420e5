"""A Workspace that grows: the status word stays, the new buffer is cleared on
the stream of the launch that needs it, and the old one goes to nobody else while
a stream still works in it."""
import pytest
import torch

from paper_2609_32831_gb300 import _lib, api


def test_the_status_word_stays():
    ws = api.Workspace("cpu")
    ws.get(256)
    ws.bufs["scratch"][:16] = torch.arange(16, dtype=torch.uint8)
    ws.get(4096)
    assert ws.bufs["scratch"].numel() == 4096
    assert ws.bufs["scratch"][:16].tolist() == list(range(16)) and not ws.bufs["scratch"][16:].any()


DEV = "cuda"
LONG = 1_000_000_000   # cycles, about half a second


def _select(ws, stream=None, bad=False):
    x = torch.randn((4, 3, 50000), generator=torch.Generator().manual_seed(1)).to(DEV)
    if bad:
        x[0, 0, 7] = float("nan")
    s = torch.zeros((4, 3), device=DEV)
    torch.cuda.synchronize()
    return lambda: api.beam_select(x, s, 8, ws=ws, stream=stream)


@pytest.mark.gpu
def test_cleared_on_the_launchs_stream():
    """With the current stream busy, a first call on another stream is done, its
    buffer cleared, before the current stream gets to anything."""
    side = torch.cuda.Stream()
    ws = api.Workspace(DEV)
    want = _select(api.Workspace(DEV))()
    call = _select(ws, side)
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn((1, h, 2000, 128), generator=g).bfloat16().to(DEV) for h in (4, 2, 2))
    out, state = api.linear_attend(q, k, v, [-0.01, -0.1], ws=api.Workspace(DEV))
    torch.cuda.synchronize()
    torch.cuda._sleep(LONG)
    got = call()
    got2 = api.linear_attend(q, k, v, [-0.01, -0.1], ws=ws, stream=side)
    side.synchronize()
    assert not torch.cuda.current_stream().query(), "the current stream is still busy"
    assert ws.status(side) == 0
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert torch.equal(got2[0], out) and torch.equal(got2[1], state)


@pytest.mark.gpu
def test_an_error_survives_growth():
    ws = api.Workspace(DEV)
    _select(ws, bad=True)()
    small = ws.bufs["scratch"].numel()
    ws.get(4 * small)
    assert ws.bufs["scratch"].numel() == 4 * small
    assert ws.status() == _lib.UC_ERR_RANGE and ws.status() == 0
    _select(ws, bad=True)()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):   # a graph's first large call: nothing of the copy goes into the graph
        ws.get(16 * small)
    assert ws.status() == _lib.UC_ERR_RANGE and ws.status() == 0
    graph.replay()
    assert ws.status() == 0


@pytest.mark.gpu
def test_the_old_buffer_waits_for_its_streams():
    side = torch.cuda.Stream()
    ws = api.Workspace(DEV)
    size = 64 << 20
    ws.get(size)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    ptr, _ = ws.get(size, stream=side)   # a launch on side works in it
    ws.get(2 * size)                     # and a later one on the current stream needs more
    other = torch.empty(size, dtype=torch.uint8, device=DEV)
    assert not side.query(), "the other stream is still busy"
    assert other.data_ptr() != ptr
    torch.cuda.synchronize()
