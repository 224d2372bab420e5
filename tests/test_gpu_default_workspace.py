"""Calls that are given no workspace, on two streams at once: neither works in
the other's scratch."""
import pytest
import torch

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import api  # noqa: E402

DEV = "cuda"


def _randn(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return lambda *s: torch.randn(s, generator=g, device=DEV)


def _window(B, hq, hkv, T, n, window):
    """Prompts: T queries, the last of n tokens."""
    def make(seed):
        r = _randn(seed)
        q, k, v = (r(B, h, x, 128).bfloat16() for h, x in ((hq, T), (hkv, n), (hkv, n)))
        cache, lengths = uc.WindowCache(k, v, window, 3), torch.full((B,), n, dtype=torch.int32, device=DEV)
        return lambda **kw: uc.window_attend(q, cache, lengths, **kw)
    return make


def _verify(seed):
    r = _randn(seed)
    x, y = r(64, 4, 50001), r(64, 3, 50001)
    tokens = y.argmax(dim=-1).int()
    u, e = r(64, 3).sigmoid(), r(64, 50001).exp()
    return lambda **kw: uc.verify_draft(x, tokens, u=u, noise=e, draft_logits=y, **kw)


def _linear(seed):
    r = _randn(seed)
    q, k, v = (r(2, h, 9000, 128).bfloat16() for h in (8, 4, 4))
    return lambda **kw: uc.linear_attend(q, k, v, [-0.01] * 4, **kw)


def _beam(seed):
    r = _randn(seed)
    x, s = r(32, 4, 50001), r(32, 4)
    return lambda **kw: uc.beam_select(x, s, 8, **kw)


CASES = {"prompt": _window(1, 16, 16, 5000, 9000, 3000),         # more items than SMs
         "ranges": _window(8, 8, 1, 9, 9000, 1 << 30),           # keys split: parts and their join
         "drafts": _verify, "linear": _linear, "beams": _beam}


@pytest.mark.parametrize("case", CASES, ids=list(CASES))
def test_two_streams_at_once(case):
    calls = [CASES[case](seed) for seed in (1, 2)]
    want = [[x.clone() for x in c(ws=uc.Workspace(DEV))] for c in calls]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for c, s in zip(calls, streams):      # (workspaces as large as they get)
        c(stream=s)
    torch.cuda.synchronize()
    got = [[], []]
    for s in streams:
        with torch.cuda.stream(s):
            torch.cuda._sleep(40_000_000)  # both queues fill meanwhile
    for _ in range(6):
        for i in range(2):
            got[i].append(calls[i](stream=streams[i]))
    torch.cuda.synchronize()
    assert api.default_workspace(DEV).status() == 0
    for i in range(2):
        for g in got[i]:
            for a, b in zip(g, want[i]):
                assert torch.equal(a, b)
