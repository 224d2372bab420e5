"""Drafts of several tokens, up to 128 query rows of a KV head, are attended as exactly as single
tokens: probabilities enter the product with 16 bits, so outputs carry their own rounding and no
other. Against fp64, and against the same tokens decoded one by one."""
import numpy as np
import pytest
import torch

from oracle import window as owin
from tests.test_gpu_rotary import rows
from tests.test_gpu_window import check, ints, make_cache

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import _lib  # noqa: E402

DEV = "cuda"

# B, hq, hkv, T, window, sinks, rows, lengths, n_query
DRAFTS = [
    (16, 16, 2, 5, 200, 4, 208, [150 + 40 * b for b in range(16)], None),       # 40 rows; rings
    (3, 7, 1, 18, 120, 3, 300, [250, 18, 300], [18, 18, 7]),                    # 126 rows
    (2, 8, 1, 16, 90, 20, 140, [1000, 139], None),                              # 128; more first tokens than 16
    (1, 4, 4, 128, 64, 5, 200, [200], None),                                    # a head alone
    (40, 16, 8, 9, 150, 2, 200, [40, 180, 9, 200, 0, 100, 3, 60] * 5, None),    # more items than SMs
    (1, 8, 1, 9, 1 << 30, 5, 700, [690], None),                                 # keys split over ranges
]


@pytest.mark.parametrize("B,hq,hkv,T,window,sinks,n_rows,lengths,n_query", DRAFTS)
@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
def test_as_exact_as_single_tokens(B, hq, hkv, T, window, sinks, n_rows, lengths, n_query, layout):
    g = torch.Generator(device=DEV).manual_seed(window + T)
    k, v = make_cache(g, B, hkv, n_rows, lengths, sinks, layout == "bthd")
    q = rows(g, B, hq, T, layout)
    ws = uc.Workspace(DEV)
    out, lse = uc.window_attend(q, uc.WindowCache(k, v, window, sinks), ints(lengths),
                                None if n_query is None else ints(n_query), ws=ws)
    want = owin.attend(q.float().cpu().numpy(), k.float().cpu().numpy(), v.float().cpu().numpy(), lengths,
                       [T] * B if n_query is None else n_query, window, sinks)
    assert ws.status() == _lib.UC_OK
    check(out, lse, want, True)


@pytest.mark.parametrize("B,hq,hkv,T,n", [(1, 8, 1, 12, 3000), (80, 8, 2, 12, 600)])
@pytest.mark.parametrize("size", [30.0, 1000.0, 1e8])
def test_logits_that_jump(B, hq, hkv, T, n, size):
    """Logits that rise by any amount from tile to tile: the reference moves, or a row leaves what it allows."""
    g = torch.Generator(device=DEV).manual_seed(8)
    k, v = make_cache(g, B, hkv, n, [n] * B, 3)
    q = rows(g, B, hq, T, "bhtd")
    rise = torch.ones(n, device=DEV)
    for at in (70, 127, 128, 200, 255, 300, 550, 650, 2100, n - 3):
        rise[min(at, n - 1)] = size ** ((at % 7 + 1) / 7)
    k = (k.float() * rise[:, None]).bfloat16()
    for window in (1 << 30, 350):
        ws = uc.Workspace(DEV)
        out, lse = uc.window_attend(q, uc.WindowCache(k, v, window, 3), ints([n] * B), ws=ws)
        o, l, spread, reach = owin.attend(q.float().cpu().numpy(), k.float().cpu().numpy(), v.float().cpu().numpy(), [n] * B,
                                          [T] * B, window, 3)
        assert ws.status() == _lib.UC_OK
        # as check(), and 2 n / 16 sums in fp32, cut, each within 2^-23; where the logits' own rounding is no small
        # share of 1 the weights say nothing, and outputs are only within what they are made of
        d = 2.0 ** -19 * reach + 2.0 ** -20
        err = np.where(d[..., None] < 0.1, (2.5 * d[..., None] + 2.0 ** -16 + n / 8 * 2.0 ** -23) * spread,
                       2 * np.abs(v.float().cpu().numpy()).max())
        got = out.double().cpu().numpy()
        assert np.isfinite(got).all()
        assert (np.abs(got - o) <= err + 2.0 ** -8 * (np.abs(o) + err)).all()
        assert (np.abs(lse.double().cpu().numpy() - l) <= d + 2.0 ** -19 + 2.0 ** -22 * np.abs(l)).all()


def test_a_token_of_a_draft_and_alone():
    """The same query over the same keys: both within a rounding of the exact output, so two steps of bf16
    apart at most where that is no smaller than 2^-14 of what it is made of."""
    g = torch.Generator(device=DEV).manual_seed(5)
    B, hq, hkv, T, n, window = 4, 16, 2, 6, 400, 150
    k, v = make_cache(g, B, hkv, n, [n] * B, 2)
    q = rows(g, B, hq, T, "bhtd")
    cache = uc.WindowCache(k, v, window, 2)
    together, l0 = uc.window_attend(q, cache, ints([n] * B))
    for t in range(T):
        alone, l1 = uc.window_attend(q[:, :, t:t + 1].contiguous(), cache, ints([n - T + 1 + t] * B))
        x, y = together[:, :, t].double(), alone[:, :, 0].double()
        # (spread: at most the largest |v|)
        assert bool(((x - y).abs() <= 2 * 2.0 ** -8 * torch.maximum(x.abs(), y.abs()) + 2.0 ** -14 * v.abs().max().double()).all())
        assert float((l0[:, :, t] - l1[:, :, 0]).abs().max()) <= 2.0 ** -15
