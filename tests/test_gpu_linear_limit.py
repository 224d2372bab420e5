"""The chunked linear attention with a wait limit far below what its waits take:
whichever warp gives up first, the launch ends, reports UC_ERR_TIMEOUT (or
finishes, where no wait was looked at often enough), and the next calls on the
same context are right again."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import _lib  # noqa: E402

DEV = "cuda"


# whole sequences of one and seven heads; a split over tokens (the pass before); fewer tokens than slots
@pytest.mark.parametrize("B,hq,hkv,T", [(40, 4, 4, 1000), (20, 28, 4, 700), (1, 14, 2, 6000), (2, 2, 2, 100)])
@pytest.mark.parametrize("limit_ns", [1, 3000])
def test_a_short_limit_ends_and_leaves_the_context_usable(B, hq, hkv, T, limit_ns):
    g = torch.Generator(device=DEV).manual_seed(T)
    q, k, v = (torch.randn((B, h, T, 128), generator=g, device=DEV).bfloat16() for h in (hq, hkv, hkv))
    decay = [-0.01 * (j + 1) for j in range(hkv)]
    ws = uc.Workspace(DEV)
    want = uc.linear_attend(q, k, v, decay, ws=ws)
    assert ws.status() == _lib.UC_OK
    prev = uc.set_wait_limit(limit_ns)
    try:
        t0 = time.perf_counter()
        for _ in range(3):
            uc.linear_attend(q, k, v, decay, ws=ws)
        status = ws.status()
        assert time.perf_counter() - t0 < 1.0
    finally:
        uc.set_wait_limit(prev)
    assert status in (_lib.UC_OK, _lib.UC_ERR_TIMEOUT)
    for _ in range(2):
        got = uc.linear_attend(q, k, v, decay, ws=ws)
        assert ws.status() == _lib.UC_OK
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
