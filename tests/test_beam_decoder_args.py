"""BeamDecoder's refusals (no GPU): sizes and the order of calls."""
import pytest
import torch

from paper_2609_32831_gb300.beams import BeamDecoder
from paper_2609_32831_gb300.engine import CacheType, RequestCache, StreamEvict


def _cache(batch, **kw):
    return RequestCache([CacheType("doc", 64, "full")], 1, batch, "cpu", n_q_heads=4, n_kv_heads=2, **kw)


@pytest.mark.parametrize("batch,beams", [(1, 0), (1, 65), (33, 2)])
def test_numbers_of_beams(batch, beams):
    with pytest.raises(ValueError, match="at most 64"):
        BeamDecoder(_cache(batch), beams, 4)


def test_no_room_for_tokens():
    with pytest.raises(ValueError, match="max_new"):
        BeamDecoder(_cache(1), 2, 0)


def test_streaming_eviction():
    with pytest.raises(ValueError, match="streaming eviction"):
        BeamDecoder(_cache(1, gen_capacity=8, stream_evict=[StreamEvict("gen", 4)]), 2, 4)


def test_order_of_calls():
    c = _cache(1)
    d = BeamDecoder(c, 2, 4, linear_decay=[[-0.1, -0.2]])
    with pytest.raises(RuntimeError, match="prefill"):
        d.start()
    k = torch.zeros((1, 2, 64, 128), dtype=torch.bfloat16)
    c.prefill([k], [k.clone()], [None])
    with pytest.raises(RuntimeError, match="linear layer"):
        d.start()
