"""Attention with a window where a CTA of the prompt kernel comes from an item that
has key tiles to one that has none, and on: ranges of keys that a short sequence
leaves empty, sequences of no tokens, blocks of queries in front of the first
token. More items than SMs; against fp64."""
import ctypes as C

import pytest
import torch

from oracle import window as owin
from tests.test_gpu_rotary import rows
from tests.test_gpu_window import check, ints, make_cache

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import _lib  # noqa: E402

DEV = "cuda"

# B, hq, hkv, T, window, sinks, rows, lengths, whether keys are split over ranges
CASES = {
    # three ranges; a length up to 128 leaves two of them empty, up to 256 one
    "ranges": (50, 16, 2, 5, 3000, 4, 3100, [900 + 31 * b for b in range(26)] + [5, 120, 256, 300, 0, 700] * 4, True),
    "ranges, none at the end": (50, 16, 2, 5, 3000, 4, 3100, [700] * 27 + [200, 100, 2500] * 5 + [0] * 8, True),
    # a block of queries and a KV head each; lengths of 0 between full ones, n_query at its default
    "no tokens": (200, 8, 2, 20, 50, 3, 90, [90, 0, 0, 30] * 50, False),
    "no tokens at the end": (200, 8, 2, 20, 50, 3, 90, [60] * 120 + [0] * 80, False),
    # several blocks of a sequence, the first ones in front of its first token
    "negative positions": (24, 16, 4, 150, 70, 2, 260, [150, 80, 0, 20, 260, 64] * 4, False),
}


@pytest.mark.parametrize("case", CASES, ids=list(CASES))
def test_items_without_keys(case):
    B, hq, hkv, T, window, sinks, n_rows, lengths, split = CASES[case]
    g = torch.Generator(device=DEV).manual_seed(T)
    k, v = make_cache(g, B, hkv, n_rows, lengths, sinks)
    q = rows(g, B, hq, T, "bhtd")
    cache = uc.WindowCache(k, v, window, sinks)
    part = B * hq * T * (128 + 4) * 4   # bytes of one range's parts
    assert (_lib.lib().uc_window_workspace_size(C.byref(cache.c), hq, T) > 2 * part) == split
    ws = uc.Workspace(DEV)
    outs = [uc.window_attend(q, cache, ints(lengths), ws=ws) for _ in range(3)]
    assert ws.status() == _lib.UC_OK
    want = owin.attend(q.float().cpu().numpy(), k.float().cpu().numpy(), v.float().cpu().numpy(), lengths, [T] * B, window,
                       sinks)
    check(*outs[0], want, False)
    for again in outs[1:]:
        assert torch.equal(again[0], outs[0][0]) and torch.equal(again[1], outs[0][1])
