"""BeamDecoder on the GPU: a small model of attention layers over compressed
caches and linear layers, its beams against the same tokens decoded one
sequence at a time through RequestCache.decode_step and linear_attend, where
nothing is selected, copied or reordered.

Tolerance of a score. A layer's output is rounded to bf16 (relative 2^-9 at
most), so a logit, a sum of such outputs with a unit-variance result, moves by
at most about 2^-9 / sqrt(3) of its rms per path, 5 standard deviations of
that in any of the vocabulary: 0.0057 per path; a log probability moves by at
most twice a logit's change, in two paths, once per token: STEPS * 2 * 2 *
0.0057. A beam that follows the wrong parent is off by the spread of a logit,
about 1 per token."""
import pytest
import torch

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300.beams import BeamDecoder  # noqa: E402
from paper_2609_32831_gb300.engine import CacheType, RequestCache  # noqa: E402

DEV = "cuda"
HQ, HKV, D, N_ATT, N_LIN, STEPS = 8, 2, 128, 2, 2, 7
TOL = STEPS * 2 * 2 * 0.0057


class Model:
    """Tokens map to q, k, v of every layer by tables; the logits are a random
    projection of the layers' outputs."""

    def __init__(self, vocab, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device=DEV)
        L = N_ATT + N_LIN
        self.V = vocab
        self.q = (2 * rand(L, vocab, HQ, D)).bfloat16()
        self.k = rand(L, vocab, HKV, D).bfloat16()
        self.v = rand(L, vocab, HKV, D).bfloat16()
        self.w = rand(L, HQ * D, vocab) / (L * HQ * D) ** 0.5
        self.decay = [[-0.02, -0.3], [-0.1, -1.0]]

    def rows(self, table, layer, tokens):  # [S, T] -> [S, H, T, 128]
        return table[layer][tokens].transpose(1, 2).contiguous()

    def logits(self, outs):  # per layer [S, HQ, 1, 128] -> [S, V], each layer's output at unit size
        x = 0
        for l, o in enumerate(outs):
            o = o.float().reshape(o.shape[0], -1)
            x = x + (o / o.square().mean(1, keepdim=True).sqrt().clamp_min(1e-3)) @ self.w[l]
        return x


def _prefilled(m, prompt, types, gen_capacity):
    B, N = prompt.shape
    c = RequestCache(types, N_ATT, B, DEV, n_q_heads=HQ, n_kv_heads=HKV, window=16, gen_capacity=gen_capacity)
    k = [m.rows(m.k, l, prompt) for l in range(N_ATT)]
    v = [m.rows(m.v, l, prompt) for l in range(N_ATT)]
    c.prefill(k, v, [m.rows(m.q, l, prompt[:, -16:]) for l in range(N_ATT)])
    return c


def _types(n):
    a, b, c = n // 2, n // 4, n - n // 2 - n // 4
    return [CacheType("doc", a, "quant", bits=4), CacheType("tools", b, "evict", keep_frac=0.5),
            CacheType("chat", c, "full")]


def _beams(m, prompt, K, cut, eos=-1, stream=None):
    B, N = prompt.shape
    c = _prefilled(m, prompt, _types(N), 0)
    d = BeamDecoder(c, K, STEPS, linear_decay=m.decay, eos=eos)
    outs = [o[:, :, -1:] for o in c.decode_step([m.rows(m.q, l, prompt[:, -1:]) for l in range(N_ATT)])]
    for l in range(N_LIN):
        a = N_ATT + l
        for lo, hi in ((0, cut), (cut, N)):  # the prompt in two pieces
            t = prompt[:, lo:hi]
            o = d.linear_prompt(l, m.rows(m.q, a, t), m.rows(m.k, a, t), m.rows(m.v, a, t))
        outs.append(o[:, :, -1:])
    d.start()
    tok = d.advance(m.logits(outs)[:, None].expand(B, K, m.V).contiguous())
    for _ in range(STEPS - 1):
        t = tok.reshape(B * K, 1).long()
        outs = [d.attend(l, m.rows(m.q, l, t), m.rows(m.k, l, t)[:, :, 0].contiguous(),
                         m.rows(m.v, l, t)[:, :, 0].contiguous()) for l in range(N_ATT)]
        outs += [d.linear(l, m.rows(m.q, N_ATT + l, t), m.rows(m.k, N_ATT + l, t), m.rows(m.v, N_ATT + l, t))
                 for l in range(N_LIN)]
        tok = d.advance(m.logits(outs).reshape(B, K, m.V))
    assert c.ws.status() == 0
    return d.sequences()


def _forced(m, prompt, seq, eos):
    """Log probability of seq [B, STEPS] behind the prompts, without beams."""
    B, N = prompt.shape
    c = _prefilled(m, prompt, _types(N), STEPS)
    state = [None] * N_LIN
    outs = c.decode_step([m.rows(m.q, l, prompt[:, -1:]) for l in range(N_ATT)])
    for l in range(N_LIN):
        a = N_ATT + l
        o, state[l] = uc.linear_attend(m.rows(m.q, a, prompt), m.rows(m.k, a, prompt), m.rows(m.v, a, prompt),
                                       m.decay[l])
        outs.append(o[:, :, -1:])
    total = torch.zeros(B, dtype=torch.float64, device=DEV)
    ended = torch.zeros(B, dtype=torch.bool, device=DEV)
    for i in range(STEPS):
        lp = torch.log_softmax(m.logits(outs).double(), dim=1).gather(1, seq[:, i:i + 1])[:, 0]
        total += torch.where(ended, torch.zeros_like(lp), lp)
        ended |= seq[:, i] == eos
        if i + 1 == STEPS:
            break
        t = seq[:, i:i + 1]
        outs = c.decode_step([m.rows(m.q, l, t) for l in range(N_ATT)],
                             [m.rows(m.k, l, t)[:, :, 0].contiguous() for l in range(N_ATT)],
                             [m.rows(m.v, l, t)[:, :, 0].contiguous() for l in range(N_ATT)])
        for l in range(N_LIN):
            a = N_ATT + l
            o, state[l] = uc.linear_attend(m.rows(m.q, a, t), m.rows(m.k, a, t), m.rows(m.v, a, t), m.decay[l],
                                           state=state[l], out_state=state[l])
            outs.append(o)
    return total


@pytest.mark.parametrize("B,K,N,V,cut", [(1, 4, 300, 211, 129), (3, 5, 257, 97, 256), (2, 1, 200, 50, 7)])
def test_scores_are_those_of_the_tokens(B, K, N, V, cut):
    m = Model(V, 3 + B)
    prompt = torch.randint(0, V, (B, N), device=DEV, generator=torch.Generator(device=DEV).manual_seed(B))
    seq, score = _beams(m, prompt, K, cut)
    assert seq.shape == (B, K, STEPS) and bool((score[:, :-1] >= score[:, 1:]).all())
    for i in range(K):
        assert (_forced(m, prompt, seq[:, i], -1) - score[:, i].double()).abs().max().item() <= TOL
    for b in range(B):
        assert len({tuple(s.tolist()) for s in seq[b]}) == K, "two beams hold the same tokens"


def test_finished_beams_keep_their_scores():
    B, K, N, V, eos = 2, 6, 180, 5, 2  # (a small vocabulary: the end token is chosen early)
    m = Model(V, 11)
    prompt = torch.randint(0, V, (B, N), device=DEV, generator=torch.Generator(device=DEV).manual_seed(5))
    seq, score = _beams(m, prompt, K, 100, eos=eos)
    ends = (seq == eos).any(2)
    assert bool(ends.any()), "inputs in which a beam ends"
    for i in range(K):
        assert (_forced(m, prompt, seq[:, i], eos) - score[:, i].double()).abs().max().item() <= TOL
        for b in range(B):
            t = seq[b, i].tolist()
            if eos in t:
                assert all(x == eos for x in t[t.index(eos):])


def test_on_another_stream():
    m = Model(60, 4)
    prompt = torch.randint(0, 60, (2, 150), device=DEV, generator=torch.Generator(device=DEV).manual_seed(9))
    want = _beams(m, prompt, 3, 64)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _beams(m, prompt, 3, 64)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
