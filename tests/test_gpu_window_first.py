"""A layer whose first tokens are as many as the cache has rows, or more: short prompts of
a layer that keeps many."""
import numpy as np
import pytest
import torch

from oracle import window as owin
from tests.test_gpu_window import check, ints, make_cache, rows

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import _lib  # noqa: E402

DEV = "cuda"


@pytest.mark.parametrize("B,hq,hkv,T,window,sinks,n_rows,lengths,n_query", [
    (2, 4, 2, 1, 3, 20, 20, [20, 7], None),
    (2, 4, 2, 1, 1, 1 << 30, 1, [1, 0], [1, 0]),
    (3, 4, 4, 5, 2, 100, 33, [33, 5, 20], [5, 5, 0]),
    (2, 14, 2, 4, 7, 21, 20, [20, 19], None),
    (2, 4, 4, 40, 5, 100, 41, [41, 40], [40, 11]),
    (1, 28, 4, 300, 64, 2 ** 31 - 1, 300, [300], None),
    (2, 16, 16, 200, 16, 300, 300, [300, 250], None),
    (1, 8, 1, 70, 20, 4000, 3000, [2999], None)])
def test_attend(B, hq, hkv, T, window, sinks, n_rows, lengths, n_query):
    g = torch.Generator(device=DEV).manual_seed(window + T)
    k, v = make_cache(g, B, hkv, n_rows, lengths, sinks)
    q, ws = rows(g, B, hq, T, "bhtd"), uc.Workspace(DEV)
    out, lse = uc.window_attend(q, uc.WindowCache(k, v, window, sinks), ints(lengths),
                                None if n_query is None else ints(n_query), ws=ws)
    want = owin.attend(q.float().cpu().numpy(), k.float().cpu().numpy(), v.float().cpu().numpy(), lengths,
                       [T] * B if n_query is None else n_query, window, sinks)
    assert ws.status() == _lib.UC_OK
    check(out, lse, want, hq // hkv * T <= 8)


@pytest.mark.parametrize("T", [1, 3, 50])
def test_longer_sequences_count_a_first_token_less(T):
    """Beyond the rows the last one is a ring."""
    g = torch.Generator(device=DEV).manual_seed(T)
    k, v = make_cache(g, 2, 2, 60, [61, 500], 59)
    q, n = rows(g, 2, 4, T, "bhtd"), ints([61, 500])
    one = uc.window_attend(q, uc.WindowCache(k, v, 9, 59), n)
    for sinks in (60, 1000):
        for a, b in zip(one, uc.window_attend(q, uc.WindowCache(k, v, 9, sinks), n)):
            assert torch.equal(a, b)


def test_append():
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (rows(g, 2, 2, 12, "bhtd") for _ in range(2))
    kn, vn = (rows(g, 2, 2, 8, "bhtd") for _ in range(2))
    before = [x.float().cpu().numpy() for x in (k, v)]
    ws = uc.Workspace(DEV)
    total, _ = uc.window_append(uc.WindowCache(k, v, 3, 100), kn, vn, ints([4, 0]), ws=ws)
    assert ws.status() == _lib.UC_OK and total.tolist() == [12, 8]
    want = owin.append(*before, kn.float().cpu().numpy(), vn.float().cpu().numpy(), [4, 0], [8, 8], 100)
    for x, y in zip((k, v), want):
        assert np.array_equal(x.float().cpu().numpy(), y)
