"""Positions, window layers and drafts on a given stream: new outputs lie neither in
memory that work queued on the current stream still uses, nor in memory that the
current stream still reads; calls on two streams at once do not disturb each other;
the same with NaN in a row that a prompt's queries see."""
import pytest
import torch

from tests.test_gpu_rotary import freqs_of

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")

DEV = "cuda"
LONG = 1_000_000_000   # cycles, about half a second


def _of(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randn(s, generator=g).bfloat16().to(DEV)


def _i32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _rotary():
    r = _of(3)
    q, k, table, at = r(2, 4, 500, 128), r(2, 2, 500, 128), uc.Rotary(freqs_of(64)), _i32(7, 70000).view(2, 1)
    call = lambda stream: uc.rotary(table, at, q, k, stream=stream)
    return call, [lambda: torch.ones_like(q), lambda: torch.ones_like(k)]


def _append():
    r = _of(4)
    q, k, v, held, ws = r(2, 4, 300, 128), r(2, 2, 300, 128), r(2, 2, 300, 128), _i32(11, 12), uc.Workspace(DEV)
    cache = uc.WindowCache(r(2, 2, 400, 128), r(2, 2, 400, 128), 100, 4)
    call = lambda stream: uc.window_append(cache, k, v, held, rotary=uc.Rotary(freqs_of(64)), q=q, ws=ws, stream=stream)
    return call, [lambda: torch.ones_like(held), lambda: torch.ones_like(q)]


def _attend(tokens):
    r = _of(tokens)
    q, ws = r(2, 4, tokens, 128), uc.Workspace(DEV)
    cache = uc.WindowCache(r(2, 2, 1500, 128), r(2, 2, 1500, 128), 700, 4)
    n = _i32(1400, 1111)
    call = lambda stream: uc.window_attend(q, cache, n, ws=ws, stream=stream)
    return call, [lambda: torch.ones_like(q), lambda: torch.ones((2, 4, tokens), device=DEV)]


def _verify():
    r = _of(6)
    x, y = r(64, 4, 5000).float(), r(64, 3, 5000).float()
    g = torch.Generator().manual_seed(7)
    tokens = torch.randint(0, 5000, (64, 3), generator=g, dtype=torch.int32).to(DEV)
    u, e = torch.rand((64, 3), generator=g).to(DEV), torch.rand((64, 5000), generator=g).add_(0.01).to(DEV)
    ws = uc.Workspace(DEV)
    call = lambda stream: uc.verify_draft(x, tokens, u=u, noise=e, draft_logits=y, ws=ws, stream=stream)
    return call, [lambda: torch.ones(64, dtype=torch.int32, device=DEV),
                  lambda: torch.ones((64, 4), dtype=torch.int32, device=DEV), lambda: torch.ones((64, 4), device=DEV)]


CASES = [_rotary, _append, lambda: _attend(1), lambda: _attend(40), lambda: _attend(1000), _verify]
IDS = ["rotary", "append", "step", "ranges", "prompt", "verify"]


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_outputs_and_queued_work_share_no_memory(case):
    side = torch.cuda.Stream()
    call, like = case()
    want = call(None)
    for busy in (False, True):               # (once without: memory from the driver may wait for the device)
        torch.cuda.synchronize()
        if busy:
            torch.cuda._sleep(LONG)
        old = [make() for make in like]      # queued behind the sleep, then copied, then free for the allocator
        copies = [x.clone() for x in old]
        taken = {x.data_ptr() for x in old}
        del old
        got = call(side)
        side.synchronize()
        if not busy:
            del copies, got
    assert not torch.cuda.current_stream().query(), "the current stream is still busy"
    assert not taken & {x.data_ptr() for x in got}
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for x in copies:
        assert bool((x == 1).all())


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_outputs_stay_while_the_current_stream_reads_them(case):
    side = torch.cuda.Stream()
    call, _ = case()
    want = [x.clone() for x in call(None)]
    torch.cuda.synchronize()
    first = call(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(LONG)
    read = [x.clone() for x in first]        # behind the sleep
    taken = {x.data_ptr() for x in first}
    del first
    second = call(side)
    side.synchronize()
    assert not torch.cuda.current_stream().query(), "the current stream is still busy"
    assert not taken & {x.data_ptr() for x in second}
    torch.cuda.synchronize()
    for a, b in zip(read, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("tokens", [1, 40, 1000])
def test_two_at_once(tokens):
    """Each with its own workspace, on its own stream, several calls long."""
    calls = [_attend(tokens)[0], _attend(tokens)[0]]
    want = [[x.clone() for x in c(None)] for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(4):
        for i in range(2):
            got[i].append(calls[i](streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            for a, b in zip(g, want[i]):
                assert torch.equal(a, b)


@pytest.mark.parametrize("tokens", [1, 40, 600])
def test_nan_that_queries_see_is_theirs_alone(tokens):
    """A NaN in a key's or value's row reaches the queries that see it, in the channels it
    is in where it is a value's, and no others."""
    r = _of(9)
    q, k, v = r(1, 4, tokens, 128), r(1, 2, 800, 128), r(1, 2, 800, 128)
    n, at, window = _i32(700), 690, 100
    clean, clean_lse = uc.window_attend(q, uc.WindowCache(k, v, window, 2), n)
    first = 700 - tokens
    sees = torch.tensor([at <= first + t < at + window for t in range(tokens)], device=DEV)
    v2 = v.clone()
    v2[0, 1, at, 5] = float("nan")
    out, lse = uc.window_attend(q, uc.WindowCache(k, v2, window, 2), n)
    hit = torch.zeros_like(clean, dtype=torch.bool)
    hit[0, 2:, :, 5] = sees
    assert torch.equal(torch.isnan(out), hit)
    # Rows that a tile's product left NaN come from the definition: P is not rounded there (2^-8
    # of the values' weighted mean), and each result is (half a step, 2^-8 of it, at the next power of two).
    both = out[~hit].double(), clean[~hit].double()
    assert float((both[0] - both[1]).abs().max()) <= 3 * 2.0 ** -8 * float(v.abs().max())
    assert torch.equal(lse, clean_lse)
    k2 = k.clone()
    k2[0, 0, at, 9] = float("nan")
    out, lse = uc.window_attend(q, uc.WindowCache(k2, v, window, 2), n)
    hit = torch.zeros((1, 4, tokens), dtype=torch.bool, device=DEV)
    hit[0, :2] = sees
    assert torch.equal(torch.isnan(out).all(-1), hit) and torch.equal(torch.isnan(out).any(-1), hit)
    assert torch.equal(torch.isnan(lse), hit)
    assert torch.equal(out[~hit], clean[~hit])
