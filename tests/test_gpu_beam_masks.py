"""uc_beam_select over logits with large finite masks (the type's lowest value
and others that generation code uses for -inf), and with large positive values,
against the fp64 oracle.

A row's masked logits add nothing to its sum next to any other, and count alike
where nothing else is there. Tolerances: scores of tokens that are not masked
as in test_gpu_beams, with the values' magnitudes those of such tokens (2^-20 +
4 * 2^-24 * (2 |x| + |score| + 20)); a masked token's score is its distance to
the row's largest logit, three fp32 roundings: 2^-22 of it."""
import numpy as np
import pytest
import torch

from oracle import beams as obeams

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
DEV = "cuda"
LOW = {torch.float32: torch.finfo(torch.float32).min, torch.bfloat16: torch.finfo(torch.bfloat16).min,
       torch.float16: torch.finfo(torch.float16).min}
CASES = [(torch.float32, m) for m in (LOW[torch.float32], -1e30, -1e12, -1e10, -5e9, -1e9, -1e4)] + \
        [(torch.bfloat16, m) for m in (LOW[torch.bfloat16], -1e30, -1e10, -5e9)] + \
        [(torch.float16, LOW[torch.float16])]
PATTERNS = 8


def _rows(V, dtype, mask, seed):
    """One row per pattern of what is masked; row 4 holds nothing else, rows 6
    and 7 hold large positive values."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((PATTERNS, V), generator=g) * 2.5
    i = torch.arange(V)
    few = torch.randperm(V, generator=g)[:min(V, 12)]
    x[0, ~torch.isin(i, few)] = mask                 # all but a few
    x[1, (i // 4) % 2 == 0] = mask                   # aligned runs of four
    x[2, i < V // 2] = mask                          # the first half, whole tiles of it
    x[3, i >= V - V // 3] = mask                     # the end
    x[4] = mask                                      # the whole row
    x[5, torch.rand(V, generator=g) < 0.9] = mask
    x[5, V // 2] = 1.0
    x[6, (i // 4) % 2 == 0] = mask
    x[6, [V // 3, V - 1]] = -mask                    # two large ones
    x[7] = 3e4
    return x.to(dtype)


def _compare(got, ref, f, shift, mask):
    x0, s = got[0].double().cpu().numpy(), ref[0][f] + shift[:, None]
    np.testing.assert_array_equal(got[2].cpu().numpy(), ref[2][f])
    assert not got[1].any()
    assert np.isfinite(x0).all()
    masked = s <= mask / 2
    tol = np.where(masked, 2.0 ** -22 * np.abs(s), 2.0 ** -20 + 4 * 2.0 ** -24 * (2 * 3e4 * (f == 7)[:, None] + 30 + 20))
    assert (np.abs(x0 - s) <= tol).all(), (x0 - s)[np.abs(x0 - s) > tol]


# rows of one round, rows cut into tiles, and as many long rows as stay in one piece over several rounds
@pytest.mark.parametrize("V,rows", [(7, PATTERNS), (200, PATTERNS), (8193, PATTERNS), (40001, PATTERNS), (40003, 160)])
@pytest.mark.parametrize("dtype,mask", CASES)
def test_masked_rows(dtype, mask, V, rows):
    x = _rows(V, dtype, mask, V)
    n = 4
    ref = obeams.beam_select(x[:, None].double().numpy(), np.zeros((PATTERNS, 1)), n)
    f = np.arange(rows) % PATTERNS
    scores = -torch.arange(rows, dtype=torch.float32) / 16
    ws = uc.Workspace(DEV)
    got = uc.beam_select(x[f][:, None].contiguous().to(DEV), scores[:, None].to(DEV), n, ws=ws)
    assert ws.status() == 0
    _compare(got, ref, f, scores.double().numpy(), float(torch.tensor(mask).to(dtype)))


@pytest.mark.parametrize("dtype,mask", CASES)
def test_a_masked_beam_stays_behind(dtype, mask):
    """A beam of which a part is masked does not win places that are not its own."""
    V, n = 3001, 8
    g = torch.Generator().manual_seed(1)
    x = (torch.randn((2, 3, V), generator=g) * 2.5)
    x[:, 1, (torch.arange(V) // 4) % 3 > 0] = mask
    x = x.to(dtype)
    scores = torch.tensor([[0.0, -2.0, -0.3], [-0.5, -0.1, -1.0]])
    ref = obeams.beam_select(x.double().numpy(), scores.double().numpy(), n)
    tol = 2.0 ** -20 + 4 * 2.0 ** -24 * (2 * 15 + 3 + 20)
    assert ref[4].min() > 2 * tol, "inputs whose order rounding could change"
    got = uc.beam_select(x.to(DEV), scores.to(DEV), n)
    np.testing.assert_array_equal(got[1].cpu().numpy(), ref[1])
    np.testing.assert_array_equal(got[2].cpu().numpy(), ref[2])
    assert np.abs(got[0].double().cpu().numpy() - ref[0]).max() <= tol
