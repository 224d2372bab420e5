"""Long rows and long prompts: what the small cases do not reach.

Selection over rows that a CTA takes in several rounds, in every order that
changes how many candidates a round finds; scores as in test_gpu_beams
(2^-20 + 4 * 2^-24 of the values' magnitudes).

States of long prompts with slow decays. A chunk's own sum takes 24 additions
in the tensor cores (8 slices of 16 tokens, three parts each), each of which may
cut below one unit in the last place, 2^-23 of the running sum; the chunks'
sums are added in fp32, with 2^-24 for each of the few roundings per chunk
that the decay has not forgotten. Cuts go one way, so they add up over chunks in
proportion: 24 * 2^-23 + 8 * 2^-24 of the state's norm."""
import numpy as np
import pytest
import torch

from oracle import beams as obeams

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
DEV = "cuda"
STATE_TOL = 24 * 2.0 ** -23 + 8 * 2.0 ** -24


def _patterns(V, g):
    i = torch.arange(V, dtype=torch.float32)
    ninf = torch.full((V,), float("-inf"))
    noise = torch.randn(V, generator=g) * 2.5
    at = lambda f: int(V * f)
    one = ninf.clone()
    one[-1] = 0.5
    rows = [i / V * 20 - 10, 10 - i / V * 20, torch.zeros(V), torch.cat([ninf[:at(.45)], torch.zeros(V - at(.45))]),
            torch.floor(i / 3000), torch.cat([noise[:at(.7)], noise[at(.7):] + 5]),
            torch.cat([ninf[:at(.6)], i[at(.6):] / V]), noise, one, (i % 4096) / 512, ninf]
    return torch.stack(rows)


@pytest.mark.parametrize("dtype,V", [(torch.float32, 40003), (torch.bfloat16, 100003), (torch.float16, 65536)])
@pytest.mark.parametrize("n", [1, 7, 32])
def test_rows_of_several_rounds(dtype, V, n):
    rows = _patterns(V, torch.Generator().manual_seed(V + n)).to(dtype)
    B = 160  # (as many rows as keep a row in one piece)
    x = rows.repeat((B + len(rows) - 1) // len(rows), 1)[:B, None].contiguous()
    scores = -torch.arange(B, dtype=torch.float32)[:, None] / 16
    ws = uc.Workspace(DEV)
    got = [t.cpu().numpy() for t in uc.beam_select(x.to(DEV), scores.to(DEV), n, ws=ws)]
    assert ws.status() == 0
    ref = obeams.beam_select(rows[:, None].double().numpy(), np.zeros((len(rows), 1)), n)
    f = np.arange(B) % len(rows)
    np.testing.assert_array_equal(got[2], ref[2][f])
    assert (got[1] == 0).all() and not got[3].any()
    want = ref[0][f] + scores.double().numpy()
    assert np.array_equal(np.isneginf(got[0]), np.isneginf(want))
    fin = np.isfinite(want)
    tol = 2.0 ** -20 + 4 * 2.0 ** -24 * (2 * 20 + 10 + 20)
    assert np.abs(got[0][fin] - want[fin]).max() <= tol


def test_rows_of_several_rounds_with_values_that_are_no_logits():
    V, B = 40003, 160
    x = torch.randn((B, 1, V), generator=torch.Generator().manual_seed(1))
    ws = uc.Workspace(DEV)
    clean = x.clone()
    for b, (at, bad) in enumerate([(0, float("nan")), (39999, float("inf")), (20000, float("nan"))]):
        x[7 * b, 0, at] = bad
        clean[7 * b, 0, at] = float("-inf")
    scores = torch.zeros((B, 1), device=DEV)
    got = uc.beam_select(x.to(DEV), scores, 5, ws=ws)
    assert ws.status() == 4  # UC_ERR_RANGE
    want = uc.beam_select(clean.to(DEV), scores, 5, ws=ws)
    assert ws.status() == 0
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def _state64(k, v, g):
    T = k.shape[0]
    w = torch.exp(g * torch.arange(T - 1, -1, -1, dtype=torch.float64, device=DEV))
    return (k.double() * w[:, None]).T @ v.double()


@pytest.mark.parametrize("B,hq,T", [(1, 2, 16384), (1, 14, 8000), (32, 2, 4096)])  # runs; parts of heads; whole sequences
def test_states_of_slow_decays(B, hq, T):
    hkv, decay = 2, [-1e-4, -3e-3]
    g = torch.Generator(device=DEV).manual_seed(T)
    q, k, v = (torch.randn((B, h, T, 128), generator=g, device=DEV).bfloat16() for h in (hq, hkv, hkv))
    ws = uc.Workspace(DEV)
    state = torch.randn((B, hkv, 128, 128), generator=g, device=DEV)
    out, new = uc.linear_attend(q, k, v, decay, state=state, ws=ws)
    assert ws.status() == 0
    for b in {0, B - 1}:
        for j in range(hkv):
            ref = _state64(k[b, j], v[b, j], decay[j]) + state[b, j].double() * float(np.exp(decay[j] * T))
            assert ((new[b, j].double() - ref).norm() / ref.norm()).item() <= STATE_TOL


@pytest.mark.parametrize("B,hq,hkv,T", [(8, 28, 4, 4096), (4, 16, 16, 2049), (2, 6, 2, 5000), (16, 7, 1, 1500)])
def test_many_tiles_finish_in_time_and_repeat(B, hq, hkv, T):
    """Every wait between the warps of a CTA is met by what it waits for: no
    call runs into the wait limit, whatever their order, and all agree."""
    g = torch.Generator(device=DEV).manual_seed(B)
    q, k, v = (torch.randn((B, h, T, 128), generator=g, device=DEV).bfloat16() for h in (hq, hkv, hkv))
    lengths = [T - (37 * b) % (T // 2) for b in range(B)]
    decay = [-0.5 ** (j + 1) for j in range(hkv)]
    ws = uc.Workspace(DEV)
    first = uc.linear_attend(q, k, v, decay, lengths=lengths, ws=ws)
    for _ in range(30):
        again = uc.linear_attend(q, k, v, decay, lengths=lengths, ws=ws)
    assert ws.status() == 0
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_an_overflowed_state_stays_infinite():
    k = torch.ones((1, 1, 300, 128), dtype=torch.bfloat16, device=DEV)
    state = torch.zeros((1, 1, 128, 128), device=DEV)
    state[0, 0, 3, 5], state[0, 0, 4, 6] = float("inf"), float("-inf")
    _, new = uc.linear_attend(k, k, k, [-1e-3], state=state)
    assert new[0, 0, 3, 5].item() == float("inf") and new[0, 0, 4, 6].item() == float("-inf")
    new[0, 0, 3, 5] = new[0, 0, 4, 6] = new[0, 0, 0, 0]
    assert torch.isfinite(new).all()


def test_a_step_replays_from_a_graph():
    """One decoding step (a linear layer, the selection, the reorder) and a
    prompt, captured once and replayed over new inputs, equal the calls."""
    B, K, V, hq, hkv = 2, 3, 5000, 6, 2
    S = B * K
    g = torch.Generator(device=DEV).manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=g, device=DEV)
    decay = [-0.01, -0.4]
    qkv = [rand(S, h, 1, 128).bfloat16() for h in (hq, hkv, hkv)]
    prompt = [rand(B, h, 400, 128).bfloat16() for h in (hq, hkv, hkv)]
    state, moved, new = (torch.empty((n, hkv, 128, 128), device=DEV) for n in (S, S, B))
    logits, scores = rand(B, K, V), rand(B, K)
    ws = uc.Workspace(DEV)

    def step():
        o = uc.linear_attend(*qkv, decay, state=state, out_state=state, ws=ws)[0]
        sel = uc.beam_select(logits, scores, K, eos=1, ws=ws)
        uc.reorder([(state, moved)], sel[1], ws=ws)
        p = uc.linear_attend(*prompt, decay, out_state=new, ws=ws)[0]
        return (o, *sel, p)

    start = rand(S, hkv, 128, 128)
    state.copy_(start)
    step()  # (the workspace has its size before the capture)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(3):
        for t in qkv + prompt:
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        logits.normal_(generator=g)
        state.copy_(start)
        graph.replay()
        got_now = [t.clone() for t in got] + [moved.clone(), new.clone(), state.clone()]
        state.copy_(start)
        want = [*step(), moved, new, state]
        for a, b in zip(got_now, want):
            assert torch.equal(a, b)
    assert ws.status() == 0
