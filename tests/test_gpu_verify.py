"""Verification of drafted tokens against fp64: types, strides, odd vocabularies,
banned tokens, fewer drafts, temperature 0, ties, bad inputs."""
import numpy as np
import pytest
import torch

from oracle import drafts as odraft

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import _lib  # noqa: E402

DEV = "cuda"
FAR = 1e-5  # what a probability may be off by, relative: logits' differences of up to 40 / temperature cut to 24 bits, sums of
#             a million terms in fp32 (each thread's few hundred, then trees), exp2 within 2^-22


def make(seed, B, T, V, dtype, tau, model, wide=False, spread=2.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((B, T + 1, V), generator=g, device=DEV) * spread
    y = x[:, :T] + 0.5 * torch.randn((B, T, V), generator=g, device=DEV)
    ban = torch.rand((B, T + 1, V), generator=g, device=DEV) < 0.02
    ban[..., 0] = False
    x, y = (z.masked_fill(ban[:, :z.shape[1]], -float("inf")).to(dtype) for z in (x, y))
    if wide:       # rows apart, and behind an offset
        xw = torch.full((B, T + 2, V + 3), float("nan"), device=DEV, dtype=dtype)
        xw[:, 1:, 2:2 + V] = x
        yw = torch.full((B, T, V + 5), float("nan"), device=DEV, dtype=dtype)
        yw[..., 1:1 + V] = y
        x, y = xw[:, 1:, 2:2 + V], yw[..., 1:1 + V]
    source = (y if model else x[:, :T]).float()
    noise = torch.empty((B, T, V), device=DEV).exponential_(generator=g)
    tokens = (source / max(tau, 0.1) - noise.log()).argmax(dim=-1).int()
    u = torch.rand((B, T), generator=g, device=DEV)
    e = torch.empty((B, V), device=DEV).exponential_(generator=g).clamp_(min=1e-30)
    return x, y if model else None, tokens, u, e


def compare(got, x, y, tokens, u, e, n, tau):
    cpu = lambda z: None if z is None else z.double().cpu().numpy() if z.is_floating_point() else z.cpu().numpy()
    a, out, lp, margin = odraft.verify(cpu(x), cpu(tokens), cpu(u), cpu(e), cpu(y), n, tau)
    sure = margin > FAR
    assert np.array_equal(got[0].cpu().numpy()[sure], a[sure])
    assert np.array_equal(got[1].cpu().numpy()[sure], out[sure])
    ls = got[2].double().cpu().numpy()
    assert (np.abs(ls - lp)[sure] <= FAR + 2.0 ** -22 * np.abs(lp[sure])).all()
    return sure


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tau", [0.0, 0.6, 1.0, 1.5])
@pytest.mark.parametrize("B,T,V,model,wide", [(1, 1, 1, True, False), (1, 4, 32000, True, False), (7, 3, 65537, False, False),
                                              (3, 5, 1001, True, True), (2, 8, 17, False, True), (40, 2, 300, True, False)])
def test_against_fp64(B, T, V, model, wide, tau, dtype):
    x, y, tokens, u, e = make(V + T, B, T, V, dtype, tau, model, wide)
    ws = uc.Workspace(DEV)
    for n in (None, [(T + b) % (T + 1) for b in range(B)]):
        nd = None if n is None else torch.tensor(n, dtype=torch.int32, device=DEV)
        got = uc.verify_draft(x, tokens, u=u, noise=e, draft_logits=y, n_draft=nd, temperature=tau, ws=ws)
        assert ws.status() == _lib.UC_OK
        sure = compare(got, x, y, tokens, u, e, n, tau)
        assert sure.mean() >= 0.9 or V == 1
        if tau == 0:
            alone = uc.verify_draft(x, tokens, n_draft=nd, temperature=0)
            assert all(torch.equal(p, q) for p, q in zip(alone, got))


def test_a_draft_like_the_target_is_accepted():
    x, _, tokens, u, e = make(1, 4, 6, 5000, torch.bfloat16, 1.0, True)
    got = uc.verify_draft(x, tokens, u=u * 0.999, noise=e, draft_logits=x[:, :6])
    assert got[0].tolist() == [6] * 4 and torch.equal(got[1][:, :6], tokens)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [9, 70000])
def test_ties_go_to_the_lowest_token(dtype, V):
    x = torch.zeros((1, 2, V), dtype=dtype, device=DEV)
    x[0, 0, [3, V - 2]] = 1.0
    t = torch.tensor([[3]], dtype=torch.int32, device=DEV)
    assert uc.verify_draft(x, t, temperature=0)[1].tolist() == [[3, 0]]
    assert uc.verify_draft(x, t + V - 5, temperature=0)[1].tolist() == [[3, -1]]
    u, e = torch.full((1, 1), 0.999999, device=DEV), torch.ones((1, V), device=DEV)
    x[0, 0] = 0                        # equal weights, all drawn with equal noise
    assert uc.verify_draft(x, t * 0, u=u, noise=e)[1].tolist() == [[1, -1]]
    assert uc.verify_draft(x, t, u=u * 0, noise=e)[1].tolist() == [[3, 0]]


@pytest.mark.parametrize("low", [-3.0e38, -1e30, -65000.0])
def test_masks_of_the_lowest_value(low):
    """Finite masks far below every logit, and rows that are masked but for one token."""
    x, y, tokens, u, e = make(5, 3, 4, 3001, torch.float32, 0.7, True)
    x, y = (torch.where(torch.isinf(z), torch.full_like(z, low), z) for z in (x, y))
    x[1, 2] = low
    x[1, 2, 1234] = 0.5
    ws = uc.Workspace(DEV)
    got = uc.verify_draft(x, tokens, u=u, noise=e, draft_logits=y, temperature=0.7, ws=ws)
    assert ws.status() == _lib.UC_OK
    assert compare(got, x, y, tokens, u, e, None, 0.7).all()


def test_bad_inputs_are_reported():
    x, y, tokens, u, e = make(6, 3, 2, 500, torch.bfloat16, 1.0, True)
    ws = uc.Workspace(DEV)
    call = lambda **kw: uc.verify_draft(**{**dict(logits=x, tokens=tokens, u=u, noise=e, draft_logits=y, ws=ws), **kw})
    want = call()
    assert ws.status() == _lib.UC_OK
    for bad in (float("nan"), float("inf")):     # counts as -inf
        z, banned = x.clone(), x.clone()
        z[1, 0, 7], banned[1, 0, 7] = bad, -float("inf")
        got = call(logits=z)
        assert ws.status() == _lib.UC_ERR_RANGE
        assert all(torch.equal(p, q) for p, q in zip(got, call(logits=banned)))
        assert ws.status() == _lib.UC_OK
    z = x.clone()
    z[2] = -float("inf")                         # no finite logit: nothing is accepted
    got = call(logits=z)
    assert ws.status() == _lib.UC_ERR_RANGE and int(got[0][2]) == 0 and torch.equal(got[1][:2], want[1][:2])
    for t in (-1, 500, 2 ** 31 - 1):
        z = tokens.clone()
        z[0, 0] = t
        got = call(tokens=z)
        assert ws.status() == _lib.UC_ERR_RANGE and int(got[0][0]) == 0 and torch.equal(got[1][1:], want[1][1:])
        got = call(tokens=z, draft_logits=None)
        assert ws.status() == _lib.UC_ERR_RANGE and int(got[0][0]) == 0
    nd = torch.tensor([5, 2, 1], dtype=torch.int32, device=DEV)
    a = call(n_draft=nd)
    assert ws.status() == _lib.UC_ERR_RANGE
    b = call(n_draft=nd.clamp(max=2))
    assert ws.status() == _lib.UC_OK and all(torch.equal(p, q) for p, q in zip(a, b))


def test_the_same_call_gives_the_same_bits():
    x, y, tokens, u, e = make(7, 5, 5, 40001, torch.bfloat16, 1.0, True)
    first = uc.verify_draft(x, tokens, u=u, noise=e, draft_logits=y)
    for _ in range(5):
        assert all(torch.equal(p, q) for p, q in zip(first, uc.verify_draft(x, tokens, u=u, noise=e, draft_logits=y)))
