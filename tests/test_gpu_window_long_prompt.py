"""Prompts longer than the ring that keeps them: attention over their own rows, then the
append, then steps of one and of several tokens over the ring, each against fp64 over
every token so far."""
import numpy as np
import pytest
import torch

from oracle import window as owin
from tests.test_gpu_rotary import freqs_of, rows
from tests.test_gpu_window import check, ints

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import _lib  # noqa: E402

DEV = "cuda"


@pytest.mark.parametrize("hq,hkv,window,sinks,lengths", [
    (4, 2, 50, 4, [300, 1, 0, 57, 131]), (14, 2, 130, 3, [700, 130, 133, 500, 2]), (4, 4, 1, 0, [40, 9, 1, 0, 33])])
def test_a_prompt_then_steps(hq, hkv, window, sinks, lengths):
    B, T, most = len(lengths), max(lengths), 5              # steps of up to 5 tokens
    g = torch.Generator(device=DEV).manual_seed(T)
    ws, table = uc.Workspace(DEV), uc.Rotary(freqs_of(64))
    ring = [rows(g, B, hkv, sinks + window + most - 1, "bhtd") for _ in range(2)]
    for x in ring:
        x.fill_(float("nan"))
    cache = uc.WindowCache(*ring, window, sinks)
    q, k, v = (rows(g, B, h, T, "bthd") for h in (hq, hkv, hkv))
    n, zeros = ints(lengths), ints([0] * B)
    q, k = uc.rotary(table, zeros[:, None], q, k)
    out, lse = uc.window_attend(q, uc.WindowCache(k, v, window, sinks), n, n_query=n, ws=ws)
    held, _ = uc.window_append(cache, k, v, zeros, n_new=n, ws=ws)
    assert ws.status() == _lib.UC_OK and held.tolist() == lengths
    now = list(lengths)
    steps = [1, 1, 5, 1, 3, 5]
    full = [np.zeros((B, hkv, T + sum(steps), 128), np.float32) for _ in range(2)]     # a row per token
    for x, y in zip(full, (k, v)):
        x[:, :, :T] = y.float().cpu().numpy()
    host = lambda x: x.float().cpu().numpy()
    check(out, lse, owin.attend(host(q), *full, lengths, lengths, window, sinks), False)
    for t in steps:
        q, k, v = (rows(g, B, h, t, "bhtd") for h in (hq, hkv, hkv))
        turned, kt = uc.rotary(table, held[:, None], q, k)
        total, q = uc.window_append(cache, k, v, held, rotary=table, q=q, ws=ws)
        assert torch.equal(q, turned)
        out, lse = uc.window_attend(q, cache, total, ws=ws)
        assert ws.status() == _lib.UC_OK
        for b in range(B):
            for x, y in zip(full, (kt, v)):
                x[b, :, now[b]:now[b] + t] = host(y[b])
            now[b] += t
        check(out, lse, owin.attend(host(q), *full, now, [t] * B, window, sinks), hq // hkv * t <= 8)
        held = total
        assert held.tolist() == now
