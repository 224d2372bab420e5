"""A Workspace with buffers for each stream (the default one): which buffer a call gets."""
import torch

from paper_2609_32831_gb300 import api


def test_a_buffer_for_each_stream(monkeypatch):
    capturing = False
    monkeypatch.setattr(api, "_capturing", lambda stream=None: capturing)
    ws = api.Workspace("cpu", per_stream=True)
    first, second, base = (ws.get(500, handle=h)[0] for h in (5, 6, 0))
    assert len({first, second, base}) == 3
    assert ws.get(400, handle=5)[0] == first and ws.get(500, "attend", handle=5)[0] not in (first, second, base)
    ws.bufs["scratch", 6][:16] = 3
    grown = ws.get(5000, handle=6)
    assert grown[1] == 5000 and ws.bufs["scratch", 6][:16].tolist() == [3] * 16
    assert ws.get(500, handle=5)[0] == first and ws.get(500, handle=0)[0] == base
    # a graph works in a buffer that is there already, the default stream's first
    capturing = True
    assert ws.get(500, handle=9)[0] == base and ws.get(5000, handle=9)[0] == grown[0]
    assert ws.get(500, handle=5)[0] == base
    capturing = False
    assert ws.get(500, handle=9)[0] not in (first, base, grown[0])   # but an uncaptured call on its stream has its own
    assert set(ws._graphs) == {base, grown[0]}


def test_one_buffer_otherwise(monkeypatch):
    monkeypatch.setattr(api, "_capturing", lambda stream=None: False)
    ws = api.Workspace("cpu")
    assert len({ws.get(500, handle=h)[0] for h in (0, 5, 6)}) == 1
    assert api.default_workspace(torch.device("cuda", 0)).per_stream
