"""Decoding with drafts over a layer with a sliding window, the operators together:
append with rotation, attention, verification; a step captured in a graph and
replayed; given streams; workspaces that graphs share."""
import numpy as np
import pytest
import torch

from oracle import drafts as odraft
from oracle import rotary as orot
from oracle import window as owin
from tests.test_gpu_rotary import freqs_of

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import _lib  # noqa: E402

DEV = "cuda"
B, HQ, HKV, T, W, S, V = 3, 14, 2, 4, 40, 3, 1000
ROWS = S + W + T - 1


class Step:
    """A layer and a head of random weights: tokens' embeddings are q, k, v; logits are out @ w."""

    def __init__(self, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device=DEV)
        self.emb = {n: r(V, h, 128).bfloat16() for n, h in (("q", HQ), ("k", HKV), ("v", HKV))}
        self.w = r(HQ * 128, V).mul_(0.15).bfloat16()
        self.table = uc.Rotary(freqs_of(32), scale=1.1)
        self.g = g
        self.k, self.v = (torch.full((B, HKV, ROWS, 128), float("nan"), device=DEV, dtype=torch.bfloat16) for _ in range(2))
        self.cache = uc.WindowCache(self.k, self.v, W, S)
        self.ws = uc.Workspace(DEV)

    def draw(self):
        u = torch.rand((B, T - 1), generator=self.g, device=DEV)
        e = torch.empty((B, V), device=DEV).exponential_(generator=self.g).clamp_(min=1e-30)
        return u, e

    def __call__(self, tokens, held, u, e, stream=None):
        """tokens [B, T]: the last one and T - 1 drafts. -> accepted, tokens, logprob, logits, total"""
        q, k, v = (self.emb[n][tokens.long()].transpose(1, 2) for n in "qkv")
        total, q = uc.window_append(self.cache, k, v, held, rotary=self.table, q=q, ws=self.ws, stream=stream)
        out, _ = uc.window_attend(q, self.cache, total, want_lse=False, ws=self.ws, stream=stream)
        logits = (out.transpose(1, 2).reshape(B, T, HQ * 128) @ self.w).float()
        a, tok, lp = uc.verify_draft(logits, tokens[:, 1:].contiguous(), u=u, noise=e, temperature=0.8, ws=self.ws, stream=stream)
        return a, tok, lp, logits, total


def test_a_run_of_steps():
    """Rejected tokens stay in the cache until the next step writes over them."""
    m = Step()
    rng = np.random.default_rng(0)
    known = [rng.integers(0, V, 1).tolist() for _ in range(B)]      # accepted tokens, the last not yet in the cache
    held = torch.zeros(B, dtype=torch.int32, device=DEV)
    emb = {n: x.double().cpu().numpy() for n, x in m.emb.items()}
    for step in range(30):
        drafts = rng.integers(0, V, (B, T - 1))
        tokens = torch.tensor([[known[b][-1], *drafts[b]] for b in range(B)], dtype=torch.int32, device=DEV)
        u, e = m.draw()
        a, tok, lp, logits, total = m(tokens, held, u * 0.3, e)
        assert m.ws.status() == _lib.UC_OK
        # the cache from the token lists alone
        for b in range(B):
            now = known[b] + drafts[b].tolist()
            at = np.arange(len(now))
            ks = orot.rotary(emb["k"][now].transpose(1, 0, 2)[None], at, freqs_of(32), scale=1.1)
            vs = emb["v"][now].transpose(1, 0, 2)[None]
            lost = max(0, len(now) - ROWS)                          # (only what a ring still holds)
            ck, cv = owin.append(np.zeros((1, HKV, ROWS, 128)), np.zeros((1, HKV, ROWS, 128)), ks, vs, [0], [len(now)], S)
            qs = orot.rotary(emb["q"][now[-T:]].transpose(1, 0, 2)[None], at[-T:], freqs_of(32), scale=1.1)
            want, _, spread, reach = owin.attend(qs, ck, cv, [len(now)], [T], W, S)
            ref = want[0].transpose(1, 0, 2).reshape(T, -1) @ m.w.double().cpu().numpy()
            # roundings of k, q and the outputs to bf16, each at most 2^-8 (a logit of 128 products: 2 * 2^-8 * reach)
            size = np.abs(want[0]).transpose(1, 0, 2).reshape(T, -1) + spread[0].transpose(1, 0, 2).reshape(T, -1) * \
                np.repeat(4 * 2.0 ** -8 * reach[0].T, 128, axis=1)
            tol = (2.0 ** -8 * size + np.repeat(4 * 2.0 ** -8 * reach[0].T, 128, axis=1) *
                   spread[0].transpose(1, 0, 2).reshape(T, -1)) @ np.abs(m.w.double().cpu().numpy())
            assert (np.abs(logits[b].double().cpu().numpy() - ref) <= tol + 2.0 ** -7 * np.abs(ref)).all(), (step, b, lost)
        oa, otok, olp, margin = odraft.verify(logits.double().cpu().numpy(), drafts, (u * 0.3).double().cpu().numpy(),
                                              e.double().cpu().numpy(), temperature=0.8)
        sure = margin > 1e-5
        assert np.array_equal(a.cpu().numpy()[sure], oa[sure]) and np.array_equal(tok.cpu().numpy()[sure], otok[sure])
        new = tok.cpu().numpy()
        for b in range(B):
            known[b] += new[b, :int(a[b]) + 1].tolist()
        held = held + a + 1
        assert held.tolist() == [len(x) - 1 for x in known]


def test_a_step_in_a_graph():
    """Captured once, replayed on other tokens, counts and random numbers; two graphs share a workspace."""
    m, ref = Step(1), Step(1)
    rng = np.random.default_rng(1)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    bufs = [(ints(rng.integers(0, V, (B, T))), ints([0] * B), *m.draw()) for _ in range(2)]
    for x in bufs:
        m(*x)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x in bufs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(m(*x))
        graphs.append(g)
    m.k.fill_(float("nan"))
    m.v.fill_(float("nan"))
    for step in range(12):
        i = step % 2
        new = (ints(rng.integers(0, V, (B, T))), ints([3 * step, 2 * step, 4 * step]), *ref.draw())
        for to, x in zip(bufs[i], new):
            to.copy_(x)
        graphs[i].replay()
        want = ref(*new)
        for x, y in zip(outs[i], want):
            assert torch.equal(x, y)
        assert torch.equal(torch.nan_to_num(m.k), torch.nan_to_num(ref.k))
    assert m.ws.status() == _lib.UC_OK


def test_a_given_stream():
    """Everything on a stream of its own while the current one sleeps."""
    m, ref = Step(2), Step(2)
    rng = np.random.default_rng(2)
    tokens = torch.tensor(rng.integers(0, V, (B, T)), dtype=torch.int32, device=DEV)
    held = torch.tensor([7, 0, 100], dtype=torch.int32, device=DEV)
    u, e = m.draw()
    want = ref(tokens, held, u, e)
    q, k, v = (m.emb[n][tokens.long()].transpose(1, 2) for n in "qkv")
    m.ws.get(1 << 20, "scratch")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(1_000_000_000)
    total, qr = uc.window_append(m.cache, k, v, held, rotary=m.table, q=q, ws=m.ws, stream=side)
    turned, _ = uc.rotary(m.table, held[:, None], q, stream=side)
    out, _ = uc.window_attend(qr, m.cache, total, ws=m.ws, stream=side)
    got = uc.verify_draft(want[3], tokens[:, 1:].contiguous(), u=u, noise=e, temperature=0.8, ws=m.ws, stream=side)
    side.synchronize()
    assert not torch.cuda.current_stream().query(), "the current stream is still busy"
    torch.cuda.synchronize()
    assert torch.equal(total, want[4]) and torch.equal(turned, qr)
    logits = (out.transpose(1, 2).reshape(B, T, HQ * 128) @ m.w).float()
    # (rows that no token was stored in are NaN, and reach sequences that say that they hold some)
    for x, y in zip((logits, *got), (want[3], *want[:3])):
        assert torch.allclose(x, y, rtol=0, atol=0, equal_nan=True)
