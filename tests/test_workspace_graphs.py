"""The buffer that a captured call works in stays when later calls need a larger
one: its memory goes to nobody else, and its status word is still read."""
import pytest
import torch

from paper_2609_32831_gb300 import _lib, api

DEV = "cuda"


def test_the_buffer_of_a_capture_stays(monkeypatch):
    capturing = False
    monkeypatch.setattr(api, "_capturing", lambda stream=None: capturing)
    ws = api.Workspace("cpu")
    ws.get(1000, handle=7)            # once before, as warm-up
    capturing = True
    at = ws.get(1000, handle=7)
    capturing = False
    old = ws.bufs["scratch"]
    assert at == (old.data_ptr(), 1000)
    held = old.data_ptr()
    del old
    assert ws.get(1 << 20, handle=7)[0] != held
    others = [torch.empty(1000, dtype=torch.uint8) for _ in range(64)]
    assert held not in {x.data_ptr() for x in others}
    # nothing of the kind for a call that was not captured
    ws = api.Workspace("cpu")
    ws.get(1000)
    ws.get(2000)
    assert len(ws._graphs) == 0


def _randn(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return lambda *s: torch.randn(s, generator=g, device=DEV)


@pytest.mark.gpu
def test_a_graph_is_replayed_after_its_workspace_grew():
    """Logits by beams with a small scratch, captured; the same Workspace then grows; what takes
    memory afterwards keeps its values through replays, and a bad logit is still reported."""
    r = _randn(1)
    x, s = r(4, 3, 50000), r(4, 3)
    ws = api.Workspace(DEV)
    want = [y.clone() for y in api.beam_select(x, s, 8, ws=ws)]
    size = ws.bufs["scratch"].numel()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = api.beam_select(x, s, 8, ws=ws)
    ws.get(64 << 20)
    others = [torch.full((size,), 77, dtype=torch.uint8, device=DEV) for _ in range(64)]
    for _ in range(3):
        graph.replay()
    assert ws.status() == _lib.UC_OK
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(bool((z == 77).all()) for z in others)
    x[0, 0, 7] = float("nan")
    graph.replay()
    assert ws.status() == _lib.UC_ERR_RANGE and ws.status() == _lib.UC_OK
