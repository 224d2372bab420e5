"""Prompts some of whose rows are computed again from the definition (logits that jump by more
than the tiles' reference allows, NaN and infinities in values that a row's tile holds but the row
does not see), over long contexts: no wait of the other rows' pipeline runs out meanwhile, and
values that rows do see cost no second look at all their keys. Against fp64."""
import pytest
import torch

from tests.test_gpu_rotary import rows
from tests.test_gpu_window import ints

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import _lib  # noqa: E402

DEV = "cuda"
B, H, T, HELD, SINKS = 1, 16, 5120, 20000, 3   # 320 items: CTAs take several
N = HELD + T


def make(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return tuple(rows(g, B, H, n, "bhtd") for n in (T, N, N))


def attend(q, k, v, window):
    """With every wait limited to 20 ms, a hundredth of the default."""
    ws = uc.Workspace(DEV)
    prev = uc.set_wait_limit(20_000_000)
    try:
        got = uc.window_attend(q, uc.WindowCache(k, v, window, SINKS), ints([N]), ws=ws)
        status = ws.status()                  # synchronises the stream
    finally:
        uc.set_wait_limit(prev)
    return got, status


def exact(q, k, v, window, h, at):
    """Of head h, queries `at`: out, spread, lse, reach in fp64."""
    x, y, z = (r.cpu().double() for r in (q[0, h, at], k[0, h], v[0, h]))
    pos, key = HELD + at.cpu()[:, None], torch.arange(N)[None]
    see = (key <= pos) & ((pos - key < window) | (key < SINKS))
    s = (x @ y.T / 128 ** 0.5).masked_fill(~see, -float("inf"))
    reach = (x.abs() @ y.abs().T / 128 ** 0.5).masked_fill(~see, 0).amax(1)
    p = torch.softmax(s, 1)
    return tuple(r.to(DEV) for r in (p @ z, p @ z.abs(), torch.logsumexp(s, 1), reach))


def check(got, lse, want):
    """As in test_gpu_window.py: p rounded to bf16 at most, logits within 2^-20 of what they are made of."""
    o, spread, l, reach = want
    d = 2.0 ** -19 * reach + 2.0 ** -20
    err = (2 * d[:, None] + 2.0 ** -8) * spread
    assert bool(((got.double() - o).abs() <= err + 2.0 ** -8 * (o.abs() + err)).all())
    assert bool(((lse.double() - l).abs() <= d + 2.0 ** -19 + 2.0 ** -22 * l.abs()).all())


@pytest.mark.parametrize("window", [1 << 30, 6000])
def test_logits_that_jump_late(window):
    q, k, v = make(1)
    k[:, :, 17000] *= 64          # logits of about 64 x N(0, 1): beyond 2^100 of the first tile's for every eighth query
    (out, lse), status = attend(q, k, v, window)
    assert status == _lib.UC_OK
    for h in (0, 7, 15):
        at = torch.arange(h, T, 37, device=DEV)
        check(out[0, h, at], lse[0, h, at], exact(q, k, v, window, h, at))


@pytest.mark.parametrize("window", [1 << 30, 6000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_that_are_seen(window, bad):
    """A first token's value: every query has it, in the channel it is in."""
    q, k, v = make(2)
    (want, l0), status = attend(q, k, v, window)
    assert status == _lib.UC_OK
    v[:, :, 1, 44] = bad
    (out, lse), status = attend(q, k, v, window)
    assert status == _lib.UC_OK and torch.equal(lse, l0)
    hit = torch.zeros(128, dtype=torch.bool, device=DEV)
    hit[44] = True
    assert not bool(torch.isfinite(out[..., hit]).any())
    assert torch.equal(out[..., ~hit], want[..., ~hit])


@pytest.mark.parametrize("window", [1 << 30, 6000])
def test_values_that_are_not_seen(window):
    """Tokens in the middle of tiles: queries before them and past their window keep their outputs."""
    q, k, v = make(3)
    (want, l0), status = attend(q, k, v, window)
    assert status == _lib.UC_OK
    places = [15001, HELD + 77, HELD + 1500, HELD + 4000]
    clean = v.clone()
    for i, at in enumerate(places):
        v[:, :, at, 30 * i] = float("inf") if i % 2 else float("nan")
    (out, lse), status = attend(q, k, v, window)
    assert status == _lib.UC_OK and torch.equal(lse, l0)
    pos = torch.arange(HELD, N, device=DEV)
    hit = torch.zeros((T, 128), dtype=torch.bool, device=DEV)
    for i, at in enumerate(places):
        hit[:, 30 * i] = (pos >= at) & (pos - at < window)
    assert not bool(torch.isfinite(out[:, :, hit]).any()) and bool(torch.isfinite(out[:, :, ~hit]).all())
    near = sorted({t for at in places for s in (at, at + window) for t in range(s - HELD - 40, s - HELD + 40) if 0 <= t < T})
    for h in (0, 9):
        at = torch.tensor(near, device=DEV)
        o, spread, l, reach = exact(q, k, clean, window, h, at)
        keep = ~hit[at]
        d = (2.0 ** -19 * reach + 2.0 ** -20)[:, None]
        err = (2 * d + 2.0 ** -8) * spread
        far = (out[0, h, at].double() - o).abs() - (err + 2.0 ** -8 * (o.abs() + err))
        assert bool((far[keep] <= 0).all())


def test_first_tokens_that_are_seen():
    """Tens of thousands of first tokens, one of whose values is bad: seen in every tile, window or not."""
    q, k, v = make(4)
    n = ints([N])
    ws = uc.Workspace(DEV)
    cache = uc.WindowCache(k, v, 500, 24000)
    want, l0 = uc.window_attend(q, cache, n, ws=ws)
    v[:, :, 11000, 3] = float("nan")
    prev = uc.set_wait_limit(20_000_000)
    try:
        out, lse = uc.window_attend(q, cache, n, ws=ws)
        assert ws.status() == _lib.UC_OK
    finally:
        uc.set_wait_limit(prev)
    hit = torch.zeros(128, dtype=torch.bool, device=DEV)
    hit[3] = True
    assert torch.equal(lse, l0) and not bool(torch.isfinite(out[..., hit]).any())
    # (one bad value beyond the tiles that are looked at: the rows are computed again, p not rounded)
    assert float((out[..., ~hit].float() - want[..., ~hit].float()).abs().max()) <= 3 * 2.0 ** -8 * float(v[:, :, :11000].abs().max())
