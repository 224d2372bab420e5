"""Verification where a draft is turned down although target and drafter agree to rounding (u
next to 1, rows at other vector boundaries, so that their sums differ in the last bits): nothing
is left of p - q, and the next token is one of the target's all the same."""
import pytest
import torch

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import _lib  # noqa: E402

DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V", [1001, 50001])
def test_the_next_token_is_no_banned_one(V, dtype):
    B, T = 64, 4
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.randn((B, T + 1, V), generator=g, device=DEV) * 2
    x = x.masked_fill(torch.rand((B, T + 1, V), generator=g, device=DEV) < 0.05, -float("inf"))
    x[..., 0] = -float("inf")
    x = x.to(dtype)
    y = torch.empty((B, T, V + 2), dtype=dtype, device=DEV)[..., 1:1 + V].copy_(x[:, :T])
    e = torch.empty((B, V), device=DEV).exponential_(generator=g).clamp_(min=1e-30)
    tokens = x[:, :T].float().argmax(dim=-1).int()
    u = torch.full((B, T), 1 - 2.0 ** -24, device=DEV)
    ws = uc.Workspace(DEV)
    accepted, out, logprob = uc.verify_draft(x, tokens, u=u, noise=e, draft_logits=y, ws=ws)
    assert ws.status() == _lib.UC_OK
    refused = accepted < T
    assert bool(refused.any()), "no row's sums differ: this test shows nothing"
    last = out.gather(1, accepted[:, None].long())[:, 0]
    assert bool(torch.isfinite(logprob).all()) and bool((last > 0).all())
    # nothing left of p - q anywhere: drawn from p
    p = torch.softmax(x[torch.arange(B, device=DEV), accepted.long()].double(), -1) / e.double()
    best = p.gather(1, last[:, None].long())[:, 0]
    assert bool((best >= p.amax(1) * (1 - 1e-5))[refused].all())
