"""Failure handling of the chunked linear attention without a GPU fault: a test
hook withholds one load of every CTA, the waits for it give up after 20 ms, the
call reports UC_ERR_TIMEOUT, the launch ends, and the next call on the same
context equals the one before."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import _lib  # noqa: E402

DEV = "cuda"


# whole sequences with k, q, v of the first chunk and loads of later ones (nine per chunk with seven heads, three
# with one); fewer loads than slots; a prompt split over tokens: the runs' own sums
@pytest.mark.parametrize("B,hq,hkv,T,pos", [(20, 28, 4, 700, p) for p in (0, 1, 2, 12, 20)] +
                         [(40, 4, 4, 1000, p) for p in (0, 2, 7)] + [(2, 2, 2, 100, p) for p in (0, 1, 2)] +
                         [(1, 14, 2, 6000, 0), (1, 14, 2, 20000, 1)])
def test_a_withheld_load_is_reported(B, hq, hkv, T, pos):
    g = torch.Generator(device=DEV).manual_seed(T + pos)
    q, k, v = (torch.randn((B, h, T, 128), generator=g, device=DEV).bfloat16() for h in (hq, hkv, hkv))
    decay = [-0.01 * (j + 1) for j in range(hkv)]
    ws = uc.Workspace(DEV)
    want = uc.linear_attend(q, k, v, decay, ws=ws)
    assert ws.status() == _lib.UC_OK
    prev = uc.set_wait_limit(20_000_000)
    try:
        uc.debug_withhold_tile(pos)
        t0 = time.perf_counter()
        uc.linear_attend(q, k, v, decay, ws=ws)
        status = ws.status()                  # synchronises the stream
        elapsed = time.perf_counter() - t0
    finally:
        uc.set_wait_limit(prev)
        uc.debug_withhold_tile(-1)
    assert status == _lib.UC_ERR_TIMEOUT
    assert elapsed < 1.0, elapsed             # a few 20 ms limits, not a hang
    got = uc.linear_attend(q, k, v, decay, ws=ws)
    assert ws.status() == _lib.UC_OK
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
