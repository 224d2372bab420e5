"""uc_beam_select and uc_reorder on the GPU.

Selection: parents, tokens and flags equal the fp64 oracle's wherever its
neighbouring scores of different beams are further apart than rounding can
move them (asserted of every input); scores within rounding. A score is
score_b + ((x - m) - log s) in fp32: three roundings, log's own 2 ulp, and s a
sum of up to V terms each within 2^-21: 2^-20 of s, so 2^-20 + 4 * 2^-24 of
the values' magnitudes. Reordering moves bytes: everything is equal."""
import numpy as np
import pytest
import torch

from oracle import beams as obeams

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
DEV = "cuda"
NEG = float("-inf")


def _tol(x, scores):
    f = lambda a: np.abs(a[np.isfinite(a)]).max(initial=1.0)
    return 2.0 ** -20 + 4 * 2.0 ** -24 * (2 * f(x) + f(scores) + 20)


def _check(logits, scores, n, finished=None, eos=-1, **kw):
    got = uc.beam_select(logits, scores, n, finished=finished, eos=eos, **kw)
    x, sc = logits.double().cpu().numpy(), scores.double().cpu().numpy()
    ref = obeams.beam_select(x, sc, n, None if finished is None else finished.cpu().numpy(), eos)
    tol = _tol(x, sc)
    assert ref[4].min() > 2 * tol, "inputs whose order rounding could change"
    np.testing.assert_array_equal(got[1].cpu().numpy(), ref[1])
    np.testing.assert_array_equal(got[2].cpu().numpy(), ref[2])
    np.testing.assert_array_equal(got[3].cpu().numpy(), ref[3])
    s = got[0].double().cpu().numpy()
    assert np.array_equal(np.isneginf(s), np.isneginf(ref[0]))
    fin = np.isfinite(ref[0])
    assert np.abs(s[fin] - ref[0][fin]).max(initial=0.0) <= tol
    return got


def _make(seed, B, K, V, dtype, ban=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, K, V), generator=g) * 2.5
    if ban:
        x = x.masked_fill(torch.rand((B, K, V), generator=g) < ban, NEG)
    s = torch.sort(-torch.rand((B, K), generator=g) * 3, dim=1, descending=True).values
    return x.to(dtype).to(DEV), s.to(DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,K,V,n", [(1, 1, 1, 1), (1, 1, 7, 7), (3, 2, 5, 10), (2, 4, 1000, 4), (1, 8, 8192, 8),
                                     (2, 3, 8193, 6), (2, 5, 40001, 10), (1, 32, 3001, 32), (3, 1, 100003, 2)])
def test_select(dtype, B, K, V, n):
    x, s = _make(1000 * K + V + n, B, K, V, dtype)
    _check(x, s, n)


@pytest.mark.parametrize("V", [50, 8200, 30000])
def test_first_step_banned_and_finished(V):
    x, s = _make(V, 3, 4, V, torch.float32, ban=0.3)
    first = torch.full_like(s, NEG)
    first[:, 0] = 0.0
    _check(x, first, 4)
    fin = torch.tensor([[1, 0, 0, 1], [1, 1, 1, 1], [0, 0, 0, 0]], dtype=torch.bool, device=DEV)
    _check(x, s, 8, finished=fin, eos=V - 1)
    _check(x, s, 8, finished=fin, eos=0)
    _check(x, s, 8, finished=fin.to(torch.uint8), eos=V // 2)
    # rows without a single token left, and beams that are all dead
    x[0, 1] = NEG
    x[1] = NEG
    _check(x, s, 8)
    _check(x, torch.full_like(s, NEG), 8)


@pytest.mark.parametrize("V", [33, 9000, 20000])
@pytest.mark.parametrize("n", [1, 8, 32])
def test_ties_go_by_beam_then_token(V, n):
    """All logits and scores equal, signed zeros among them: the lowest beams
    and tokens. Then a few higher values, tied within and across tiles."""
    x = torch.zeros((2, 3, V), device=DEV)
    x[:, :, ::2] = -0.0
    s = torch.zeros((2, 3), device=DEV)
    sc, parent, token, fin = uc.beam_select(x, s, n)
    assert parent.cpu().tolist() == [[i // V for i in range(n)]] * 2
    assert token.cpu().tolist() == [[i % V for i in range(n)]] * 2
    x[:, 1, [V - 1, V // 2, 3]] = 2.0
    x[:, 2, [V - 2, V // 3, 5]] = 2.0
    sc, parent, token, fin = uc.beam_select(x, s, n)
    # within a beam the tie goes by token; beams 1 and 2 hold the same values at
    # other places, so their sums may round apart and either may come first
    one, two = [(1, 3), (1, V // 2), (1, V - 1)], [(2, 5), (2, V // 3), (2, V - 2)]
    rest = [(0, i) for i in range(32)]
    assert list(zip(parent[0].tolist(), token[0].tolist())) in ((one + two + rest)[:n], (two + one + rest)[:n])


def test_many_large_logits_in_one_place():
    """The best logits lie next to one another, rise towards the end, or fill a
    whole tile: the candidate lists are as long as they get."""
    V = 3 * 8192 + 5
    ramp = torch.arange(V, dtype=torch.float32, device=DEV) / 1000
    x = torch.stack([ramp, -ramp, (ramp - 12).abs(), -(ramp - 12).abs()])[None].contiguous()
    s = torch.tensor([[0.0, -0.3, -0.6, -0.85]], device=DEV)
    _check(x, s, 32)
    x = torch.full((1, 2, V), -5.0, device=DEV)
    x[0, 0, 8192:16384] = 1.0
    sc, parent, token, fin = uc.beam_select(x, s[:, :2].contiguous(), 32)
    assert token[0].tolist() == list(range(8192, 8224)) and not parent.any()


def test_strided_rows():
    """Rows of a wider buffer, starting at any element."""
    for off in range(1, 9):
        g = torch.Generator().manual_seed(off)
        wide = (torch.randn((2, 3, 9100), generator=g) * 2.5).to(torch.bfloat16).to(DEV)
        x = wide[:, :, off:off + 9001]
        wide[:, :, :off] = float("nan")
        wide[:, :, off + 9001:] = float("nan")
        ws = uc.Workspace(DEV)
        _check(x, torch.tensor([[0.0, -0.4, -0.9]] * 2, device=DEV), 6, ws=ws)
        assert ws.status() == 0


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("nan")])
def test_values_that_are_no_logits_are_reported(bad):
    x, s = _make(5, 2, 2, 9000, torch.float32)
    ws = uc.Workspace(DEV)
    x[1, 0, 8500] = bad
    sc, parent, token, _ = uc.beam_select(x, s, 4, ws=ws)
    assert ws.status() == 4      # UC_ERR_RANGE
    ref = x.clone()
    ref[1, 0, 8500] = NEG        # counts as -inf
    again = uc.beam_select(ref, s, 4, ws=ws)
    assert ws.status() == 0
    assert torch.equal(sc, again[0]) and torch.equal(token, again[2])
    x[:] = bad
    uc.beam_select(x, s, 32, ws=ws)
    assert ws.status() == 4
    s[0, 0] = bad
    uc.beam_select(ref, s, 4, ws=ws)
    assert ws.status() == 4


# ------------------------------------------------------------------ reorder

KINDS = [("evict", 16), ("evict_quant", 4), ("quant", 2), ("quant", 4)]


def _segment(kind, bits, S, hkv, keeps, cap, seed):
    """A segment compressed from random rows, sequences holding ``keeps``."""
    N = 300
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn((S, hkv, N, 128), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    sc = torch.rand((S, hkv, N), generator=g).to(DEV)
    seg = uc.Segment(kind, bits, S, hkv, N, cap, DEV)
    seg.set_keep([N] * S if kind == "quant" else keeps)
    uc.compress_segment(k, v, seg, scores=sc)
    return seg


NAMES = ["n_kept", "kept_idx", "k", "v", "k_codes", "k_params", "v_codes", "v_params"]


def _logical(seg):
    """The bytes that seg's sequences hold, per (sequence, head, array)."""
    S, H = seg.batch, seg.n_kv_heads
    n = seg.tensor("n_kept").cpu().tolist()
    out = {}
    for name in NAMES[1:]:
        t = seg.tensor(name)
        if t is None:
            continue
        blk = t.view(torch.uint8).view(S, H, -1).cpu().numpy()
        for i in range(S):
            if name == "kept_idx":
                m = 4 * n[i]
            elif name in ("k", "v"):
                m = 256 * (n[i] if seg.bits == 16 else n[i] % 32)
            elif name.endswith("codes"):
                m = n[i] // 32 * 32 * 128 * seg.bits // 8
            else:
                m = n[i] // 32 * 512
            out[name, i] = blk[i, :, :m].copy()
    return n, out


@pytest.mark.parametrize("kind,bits", KINDS)
@pytest.mark.parametrize("hkv,cap", [(4, 300), (1, 301), (3, 410)])
def test_reorder_segments(kind, bits, hkv, cap):
    G, K = 3, 4
    keeps = [[130] * K, [1] * K, [96] * K]
    seg = _segment(kind, bits, G * K, hkv, sum(keeps, []), cap, 7)
    dst = uc.Segment(kind, bits, G * K, hkv, 300, cap + 64, DEV)
    state = torch.randn((G * K, hkv, 128, 128), device=DEV)
    odd = torch.randn((G * K, 7), device=DEV)
    new_state, new_odd = torch.zeros_like(state), torch.zeros_like(odd)
    parent = torch.tensor([[3, 3, 0, 1], [0, 1, 2, 3], [2, 0, 2, 2]], dtype=torch.int32, device=DEV)
    ws = uc.Workspace(DEV)
    uc.reorder([(seg, dst), (state, new_state), (odd, new_odd)], parent, ws=ws)
    assert ws.status() == 0
    src = obeams.source_of(parent.cpu().numpy(), K)
    n0, have = _logical(seg)
    n1, got = _logical(dst)
    assert n1 == [n0[i] for i in src] == dst.n_kept()
    for (name, i), x in got.items():
        np.testing.assert_array_equal(x, have[name, int(src[i])], err_msg=f"{name} of sequence {i}")
    idx = torch.from_numpy(src).to(DEV)
    assert torch.equal(new_state, state[idx]) and torch.equal(new_odd, odd[idx])
    # attention over the target is attention over the source, sequence by sequence
    q = torch.randn((G * K, 7 * hkv, 1, 128), device=DEV).to(torch.bfloat16)
    a, lse, _ = uc.attend(q[idx], [dst])
    r, rl, _ = uc.attend(q, [seg])
    assert float((a.float() - r[idx].float()).abs().max()) <= 2.0 ** -7 * float(r.float().abs().max())
    assert torch.allclose(lse, rl[idx], rtol=1e-6, atol=1e-6)


def test_reorder_expands_a_prompt_to_its_beams():
    """n_from = 1: every beam gets its request's prompt caches; a full view's
    rows go into the caller's tensors."""
    G, K, hkv, N = 2, 3, 2, 50
    g = torch.Generator().manual_seed(0)
    k, v = (torch.randn((G, hkv, N, 128), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    view = uc.Segment.view(k, v, 5, 40)
    nk, nv = (torch.zeros((G * K, hkv, 60, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    big = uc.Segment.view(nk, nv, 7, 40)
    vit = _segment("evict_quant", 4, G, hkv, [100, 33], 128, 1)
    wide = uc.Segment("evict_quant", 4, G * K, hkv, 300, 128, DEV)
    uc.reorder([(view, big), (vit, wide)], torch.zeros((G, K), dtype=torch.int32, device=DEV))
    for i in range(G * K):
        assert torch.equal(nk[i, :, 7:47], k[i // K, :, 5:45]) and torch.equal(nv[i, :, 7:47], v[i // K, :, 5:45])
    assert not nk[:, :, :7].any() and not nk[:, :, 47:].any()
    n0, have = _logical(vit)
    n1, got = _logical(wide)
    assert n1 == [100] * 3 + [33] * 3 == wide.n_kept()
    for (name, i), x in got.items():
        np.testing.assert_array_equal(x, have[name, i // K])


def test_reorder_many_items_and_empty_segments():
    """More arrays than one launch takes, among them segments without a token."""
    S = 4
    parent = torch.tensor([[1, 0, 3, 3]], dtype=torch.int32, device=DEV)
    src = [torch.randn((S, 5 + i), device=DEV) for i in range(300)]
    dst = [torch.empty_like(x) for x in src]
    a, b = (uc.Segment("evict", 16, S, 2, 0, 33, DEV) for _ in range(2))
    uc.reorder(list(zip(src, dst)) + [(a, b)], parent)
    idx = parent[0].long()
    for x, y in zip(src, dst):
        assert torch.equal(y, x[idx])
    assert b.tensor("n_kept").tolist() == [0] * S


def test_reorder_reports_parents_out_of_range():
    S = 4
    x = torch.randn((S, 100), device=DEV)
    y = torch.zeros_like(x)
    ws = uc.Workspace(DEV)
    uc.reorder([(x, y)], torch.tensor([[1, 4], [-1, 0]], dtype=torch.int32, device=DEV), ws=ws)
    assert ws.status() == 4
    # group 0 has sources 0 and 1, group 1 sources 2 and 3; 4 and -1 are none of them
    assert torch.equal(y[0], x[1]) and not y[1].any() and not y[2].any() and torch.equal(y[3], x[2])
