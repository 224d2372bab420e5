"""uc_linear_attend against the fp64 recurrence: single tokens and prompts,
lengths from one token to several chunks, ragged batches with empty sequences,
strided rows, head layouts, strong and absent decay, states in place, and
non-finite values where no token is.

Tolerances. Outputs are bf16: each carries its own rounding, a relative error
of at most 2^-8. On the tensor cores the products' factors are rounded to bf16
once more, the decayed q.k (per token) and the state (per channel): independent
relative errors of variance 2^-16 / 3 each, weighed with the squared terms
(the oracle's var). An element is allowed its output rounding plus eight
standard deviations, the whole tensor 1.25 of the expected norm. fp32 sums add
at most 2^-12 of that. States: the update's factor enters as two bf16 parts
(2^-16 of a term), sums are fp32: 2^-15 of the terms' magnitudes per element,
1e-5 of the norm."""
import numpy as np
import pytest
import torch

from oracle import linear as olinear

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
DEV = "cuda"
U = 2.0 ** -8


def _inputs(seed, B, hq, hkv, T, layout="bhtd", state=True):
    g = torch.Generator().manual_seed(seed)

    def rows(h):
        x = torch.randn((B, T, h, 128) if layout == "bthd" else (B, h, T, 128), generator=g).to(torch.bfloat16).to(DEV)
        return x.transpose(1, 2) if layout == "bthd" else x
    q, k, v = rows(hq), rows(hkv), rows(hkv)
    s = (torch.randn((B, hkv, 128, 128), generator=g) * 4).to(DEV) if state else None
    return q, k, v, s


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _check(q, k, v, ld, s, lengths, out, state):
    ro, rs, var, size = olinear.linear_attend(_np(q), _np(k), _np(v), ld, _np(s), lengths)
    o, st = _np(out), _np(state)
    assert np.isfinite(o).all() and np.isfinite(st).all()
    sd2 = U * U / 3 * (1 + 2.0 ** -12) * var
    err = np.abs(o - ro)
    half = U * np.maximum(np.abs(o), np.abs(ro))
    assert (err <= half + 8 * np.sqrt(sd2) + 1e-30).all(), (err - half - 8 * np.sqrt(sd2)).max()
    want = np.sqrt((half ** 2 / 3 + sd2).sum())
    assert np.linalg.norm(err) <= 1.25 * want + 1e-30
    assert (np.abs(st - rs) <= 2.0 ** -15 * size + 1e-30).all()
    assert np.linalg.norm(st - rs) <= 1e-5 * np.linalg.norm(rs) + 1e-30


@pytest.mark.parametrize("hq,hkv", [(28, 4), (4, 4), (6, 2), (1, 1), (40, 1)])
@pytest.mark.parametrize("T", [1, 2, 5, 8])
def test_tokens(hq, hkv, T):
    B = 3
    ld = np.linspace(-0.7, -0.001, hkv).tolist()
    q, k, v, s = _inputs(10 * T + hq, B, hq, hkv, T)
    out, state = uc.linear_attend(q, k, v, ld, state=s)
    _check(q, k, v, ld, s, None, out, state)


@pytest.mark.parametrize("T", [9, 63, 64, 65, 127, 128, 129, 200, 256, 300, 515])
@pytest.mark.parametrize("hq,hkv,B", [(28, 4, 1), (2, 2, 2), (9, 3, 1)])
def test_prompts(hq, hkv, B, T):
    ld = np.linspace(-0.2, -0.0005, hkv).tolist()
    q, k, v, s = _inputs(T + hq, B, hq, hkv, T, layout="bthd" if T % 2 else "bhtd", state=T % 3 != 0)
    out, state = uc.linear_attend(q, k, v, ld, state=s)
    assert out.stride() == q.stride()
    _check(q, k, v, ld, s, None, out, state)


@pytest.mark.parametrize("T,lengths", [(6, [6, 0, 1, 5]), (300, [300, 0, 1, 129]), (257, [256, 128, 127, 257]),
                                       (40, [0, 0, 0, 0]), (8, [0, 0, 0, 0])])
def test_ragged_with_anything_behind_the_end(T, lengths):
    """Rows behind a sequence's end hold NaN and infinities: nothing of them
    arrives anywhere, their outputs are zero, and an empty sequence keeps its
    state bit for bit."""
    B, hq, hkv = len(lengths), 6, 2
    ld = [-0.05, -0.01]
    q, k, v, s = _inputs(T, B, hq, hkv, T)
    for b, n in enumerate(lengths):
        q[b, :, n:] = float("nan")
        k[b, :, n:] = float("inf")
        v[b, :, n:] = float("nan")
        k[b, :, n + 1:] = float("nan")
    out, state = uc.linear_attend(q, k, v, ld, state=s, lengths=lengths)
    clean = [torch.where(torch.isfinite(x), x, torch.zeros_like(x)) for x in (q, k, v)]
    _check(*clean, ld, s, lengths, out, state)
    for b, n in enumerate(lengths):
        assert not out[b, :, n:].any()
        if n == 0:
            assert torch.equal(state[b], s[b])


@pytest.mark.parametrize("T", [1, 7, 130, 300])
def test_decay_extremes(T):
    """No decay at all, hardly any, one that underflows within a chunk, and
    one that leaves each token only itself."""
    hkv = 4
    ld = [0.0, -1e-6, -3.0, -1e30]
    q, k, v, s = _inputs(77 + T, 1, hkv, hkv, T)
    out, state = uc.linear_attend(q, k, v, ld, state=s)
    _check(q, k, v, ld, s, None, out, state)


@pytest.mark.parametrize("T", [3, 150, 700])
def test_state_in_place_and_in_parts(T):
    """The state updated in place equals the one written elsewhere, bit for
    bit; a prompt in two calls continues as in one."""
    hq, hkv, B = 12, 4, 2
    ld = [-0.02, -0.1, -0.001, -0.5]
    q, k, v, s = _inputs(5 + T, B, hq, hkv, T)
    out, state = uc.linear_attend(q, k, v, ld, state=s)
    inplace = s.clone()
    out2, same = uc.linear_attend(q, k, v, ld, state=inplace, out_state=inplace)
    assert same.data_ptr() == inplace.data_ptr()
    assert torch.equal(inplace, state) and torch.equal(out2, out)
    cut = T // 3
    o1, s1 = uc.linear_attend(q[:, :, :cut], k[:, :, :cut], v[:, :, :cut], ld, state=s)
    o2, s2 = uc.linear_attend(q[:, :, cut:], k[:, :, cut:], v[:, :, cut:], ld, state=s1)
    _check(q, k, v, ld, s, None, torch.cat([o1, o2], dim=2), s2)


def test_layouts_slices_and_streams():
    """Rows inside wider buffers (a fused projection's output), a given output,
    and a stream of the caller's."""
    B, hq, hkv, T = 2, 8, 2, 140
    g = torch.Generator().manual_seed(3)
    wide = torch.randn((B, T, hq + 2 * hkv, 128), generator=g).to(torch.bfloat16).to(DEV).transpose(1, 2)
    q, k, v = wide[:, :hq], wide[:, hq:hq + hkv], wide[:, hq + hkv:]
    ld = [-0.02, -0.1]
    buf = torch.zeros((B, T, 2 * hq, 128), dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    out, state = uc.linear_attend(q, k, v, ld, out=buf[:, hq:])
    _check(q, k, v, ld, None, None, out, state)
    assert not buf[:, :hq].any()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    ws = uc.Workspace(DEV)
    out2, state2 = uc.linear_attend(q, k, v, ld, stream=st, ws=ws)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(out, out2) and torch.equal(state, state2)
    assert ws.status() == 0


def test_long_prompt_matches_its_own_parts():
    """10000 tokens (many chunks, split over the token axis) against the same
    prompt in parts of odd lengths, which the tests above hold to the oracle."""
    B, hq, hkv, T = 1, 14, 2, 10000
    ld = [-0.0005, -0.03]
    q, k, v, s = _inputs(9, B, hq, hkv, T)
    out, state = uc.linear_attend(q, k, v, ld, state=s)
    cur, at, parts = s, 0, []
    for n in (1, 333, 2048, 4097, 3521):
        o, cur = uc.linear_attend(q[:, :, at:at + n], k[:, :, at:at + n], v[:, :, at:at + n], ld, state=cur)
        parts.append(o)
        at += n
    assert at == T
    a, b = out.double(), torch.cat(parts, dim=2).double()
    # two independently rounded results of relative error 2^-8 / sqrt(3) each for the output and the factors
    assert float((a - b).norm() / b.norm()) <= 1.25 * 2 * U / 3 ** 0.5
    assert float((state - cur).double().norm() / cur.double().norm()) <= 2e-5


def test_repeats_bit_for_bit():
    q, k, v, s = _inputs(4, 2, 28, 4, 1500)
    ld = [-0.001, -0.01, -0.1, -1.0]
    first = uc.linear_attend(q, k, v, ld, state=s)
    for _ in range(5):
        again = uc.linear_attend(q, k, v, ld, state=s)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
