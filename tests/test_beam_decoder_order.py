"""BeamDecoder.linear out of turn is refused before anything is launched: a
second step or a skipped one between two selections, or one before the first,
would leave states that belong to no beam's tokens (CPU)."""
import pytest
import torch

from paper_2609_32831_gb300 import api
from paper_2609_32831_gb300.beams import BeamDecoder
from paper_2609_32831_gb300.engine import CacheType, RequestCache


@pytest.fixture
def decoder(monkeypatch):
    c = RequestCache([CacheType("doc", 64, "full")], 1, 1, "cpu", n_q_heads=4, n_kv_heads=2)
    k = torch.zeros((1, 2, 64, 128), dtype=torch.bfloat16)
    c.prefill([k], [k.clone()], [None])
    d = BeamDecoder(c, 2, 4, linear_decay=[[-0.1, -0.2], [-0.3, -0.4]])
    d.prompt_states = [torch.zeros((1, 2, 128, 128)) for _ in range(2)]
    monkeypatch.setattr(api, "reorder", lambda *a, **kw: None)
    monkeypatch.setattr(api, "linear_attend", lambda q, k, v, decay, state=None, out_state=None, ws=None: (q, state))
    monkeypatch.setattr(api, "beam_select", lambda logits, scores, n, **kw: (
        scores, torch.zeros((1, n), dtype=torch.int32), torch.zeros((1, n), dtype=torch.int32), None))
    d.start()
    return d


def test_steps_of_linear_layers(decoder):
    d = decoder
    x = torch.zeros((2, 4, 1, 128), dtype=torch.bfloat16)
    step = lambda layer: d.linear(layer, x, x[:, :2], x[:, :2])
    logits = torch.zeros((1, 2, 10))
    with pytest.raises(RuntimeError, match="between two selections"):
        step(0)                      # nothing is chosen yet
    d.advance(logits)
    step(0)
    with pytest.raises(RuntimeError, match="between two selections"):
        step(0)                      # twice
    step(1)
    d.advance(logits)
    step(1)
    d.advance(logits)                # layer 0 missed a token
    with pytest.raises(RuntimeError, match="between two selections"):
        step(0)
    step(1)
    d.start()                        # from the prompt again
    d.advance(logits)
    step(0)
    step(1)
