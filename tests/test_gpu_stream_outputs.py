"""New outputs of a call on a given stream: not in memory that work queued on the
current stream still uses, and not given away while the current stream reads
them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")

DEV = "cuda"
LONG = 1_000_000_000   # cycles, about half a second


def _linear(side):
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn((1, h, 2000, 128), generator=g).bfloat16().to(DEV) for h in (4, 2, 2))
    ws = uc.Workspace(DEV)
    call = lambda stream: uc.linear_attend(q, k, v, [-0.01, -0.1], ws=ws, stream=stream)
    like = [lambda: torch.ones_like(q), lambda: torch.ones((1, 2, 128, 128), device=DEV)]
    return call, like


def _beams(side):
    x = torch.randn((64, 4, 3000), generator=torch.Generator().manual_seed(1)).to(DEV)
    s = torch.zeros((64, 4), device=DEV)
    ws = uc.Workspace(DEV)
    call = lambda stream: uc.beam_select(x, s, 32, ws=ws, stream=stream)
    like = [lambda: torch.ones((64, 32), device=DEV), lambda: torch.ones((64, 32), dtype=torch.int32, device=DEV),
            lambda: torch.ones((64, 32), dtype=torch.int32, device=DEV), lambda: torch.ones((64, 32), dtype=torch.bool, device=DEV)]
    return call, like


@pytest.mark.parametrize("case", [_linear, _beams])
def test_outputs_and_queued_work_share_no_memory(case):
    side = torch.cuda.Stream()
    call, like = case(side)
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


@pytest.mark.parametrize("case", [_linear, _beams])
def test_outputs_stay_while_the_current_stream_reads_them(case):
    side = torch.cuda.Stream()
    call, _ = case(side)
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
