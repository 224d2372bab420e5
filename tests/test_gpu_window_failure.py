"""Failure handling of attention with a window without a GPU fault: a test hook
withholds one load of every CTA, the waits for it give up after 20 ms, the call
reports UC_ERR_TIMEOUT, the launch ends, and the next call on the same context
equals the one before."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import _lib  # noqa: E402

DEV = "cuda"


# prompts: the first K, the first V, later ones, in CTAs of one item and of several; steps: the first tile of a
# warp's, and one behind the ring's first places
@pytest.mark.parametrize("B,hq,hkv,T,n,window,pos", [(1, 4, 4, 300, 300, 64, p) for p in (0, 1, 2, 3)] +
                         [(8, 8, 8, 2000, 2000, 300, p) for p in (0, 3, 20)] + [(1, 7, 1, 100, 8000, 1 << 30, 3)] +
                         [(2, 28, 4, 1, 5000, 4000, 0), (64, 28, 4, 1, 5000, 4000, 0), (64, 28, 4, 1, 5000, 4000, 6),
                          (4, 16, 2, 5, 3000, 2000, 0), (16, 16, 2, 5, 3000, 2000, 3)])
def test_a_withheld_load_is_reported(B, hq, hkv, T, n, window, pos):
    g = torch.Generator(device=DEV).manual_seed(T + pos)
    k, v = (torch.randn((B, hkv, n, 128), generator=g, device=DEV).bfloat16() for _ in range(2))
    q = torch.randn((B, hq, T, 128), generator=g, device=DEV).bfloat16()
    cache = uc.WindowCache(k, v, window, 4)
    lengths = torch.full((B,), n, dtype=torch.int32, device=DEV)
    ws = uc.Workspace(DEV)
    want = uc.window_attend(q, cache, lengths, ws=ws)
    assert ws.status() == _lib.UC_OK
    prev = uc.set_wait_limit(20_000_000)
    try:
        uc.debug_withhold_tile(pos)
        t0 = time.perf_counter()
        uc.window_attend(q, cache, lengths, ws=ws)
        status = ws.status()                  # synchronises the stream
        elapsed = time.perf_counter() - t0
    finally:
        uc.set_wait_limit(prev)
        uc.debug_withhold_tile(-1)
    assert status == _lib.UC_ERR_TIMEOUT
    assert elapsed < 1.0, elapsed             # a few 20 ms limits, not a hang
    got = uc.window_attend(q, cache, lengths, ws=ws)
    assert ws.status() == _lib.UC_OK
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
