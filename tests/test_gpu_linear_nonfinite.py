"""uc_linear_attend where k or v of valid tokens holds NaN or infinities: a
token reaches itself and later ones, never an earlier one, and a value channel
never another.

The reference is the fp64 recurrence with the non-finite entries at zero; what
they reach is left out of the comparison and has to be non-finite. Tolerances
of the rest as in test_gpu_linear (an element its bf16 output rounding plus
eight standard deviations of the factors' roundings); the state's 2^-15 of the
terms' magnitudes."""
import numpy as np
import pytest
import torch

from oracle import linear as olinear
from tests.test_gpu_linear import _inputs, _np

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
U = 2.0 ** -8
NAN, INF = float("nan"), float("inf")


def _check(q, k, v, ld, s, lengths, bad, out, state):
    """bad: (sequence, KV head, token, channel) of non-finite values of v."""
    clean = v.clone()
    for b, j, t, c in bad:
        clean[b, j, t, c] = 0
    ro, rs, var, size = olinear.linear_attend(_np(q), _np(k), _np(clean), ld, _np(s), lengths)
    o, st = _np(out), _np(state)
    reach, reach_s = np.zeros(o.shape, bool), np.zeros(st.shape, bool)
    g = q.shape[1] // k.shape[1]
    for b, j, t, c in bad:
        n = q.shape[2] if lengths is None else lengths[b]
        if t < n:
            reach[b, j * g:(j + 1) * g, t:n, c] = True
            reach_s[b, j, :, c] = True
    assert not np.isfinite(o[reach]).any() and not np.isfinite(st[reach_s]).any()
    err = np.abs(o - ro)[~reach]
    half = U * np.maximum(np.abs(o), np.abs(ro))[~reach]
    assert np.isfinite(o[~reach]).all() and np.isfinite(st[~reach_s]).all()
    assert (err <= half + 8 * np.sqrt(U * U / 3 * (1 + 2.0 ** -12) * var[~reach]) + 1e-30).all()
    assert (np.abs(st - rs)[~reach_s] <= 2.0 ** -15 * size[~reach_s] + 1e-30).all()


@pytest.mark.parametrize("hq,hkv,B", [(28, 4, 1), (2, 2, 2), (6, 2, 1), (2, 1, 1)])
@pytest.mark.parametrize("T", [1, 8, 9, 128, 300, 515])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
def test_values_of_later_tokens_do_not_reach_earlier_ones(hq, hkv, B, T, value):
    ld = np.linspace(-0.2, -0.0005, hkv).tolist()
    q, k, v, s = _inputs(T + hq, B, hq, hkv, T, layout="bthd" if T % 2 else "bhtd", state=T % 3 != 0)
    bad = [(0, 0, T // 2, 5), (B - 1, hkv - 1, T - 1, 127), (0, 0, T - 1, 64), (0, hkv - 1, min(T - 1, 130), 0)]
    for b, j, t, c in bad:
        v[b, j, t, c] = value
    ws = uc.Workspace("cuda")
    out, state = uc.linear_attend(q, k, v, ld, state=s, ws=ws)
    assert ws.status() == 0
    _check(q, k, v, ld, s, None, bad, out, state)


@pytest.mark.parametrize("value", [NAN, -INF])
def test_ragged_lengths_and_strong_decays(value):
    """The last valid token, the first behind the end, and decays that leave a
    token only itself (0 times what came before is still not finite)."""
    B, hq, hkv, T = 3, 4, 4, 400
    ld = [0.0, -1e-3, -3.0, -80.0]
    lengths = [400, 0, 201]
    q, k, v, s = _inputs(3, B, hq, hkv, T)
    bad = [(0, j, 140 + 10 * j, 7 * j) for j in range(hkv)] + [(2, j, 200, 30 + j) for j in range(hkv)] + \
        [(2, j, 201, 90) for j in range(hkv)] + [(1, 0, 0, 0)]
    for b, j, t, c in bad:
        v[b, j, t, c] = value
    out, state = uc.linear_attend(q, k, v, ld, state=s, lengths=lengths)
    _check(q, k, v, ld, s, lengths, bad, out, state)


@pytest.mark.parametrize("T", [8, 300])
def test_keys_of_later_tokens_do_not_reach_earlier_ones(T):
    B, hq, hkv = 2, 6, 2
    ld = [-0.05, -0.01]
    q, k, v, s = _inputs(7, B, hq, hkv, T)
    want, _ = uc.linear_attend(q, k, v, ld, state=s)
    t = 2 * T // 3
    k[1, 1, t, 9] = NAN
    k[0, 0, t, 3] = INF
    got, state = uc.linear_attend(q, k, v, ld, state=s)
    for b, j in ((0, 0), (0, 1), (1, 0), (1, 1)):
        h = slice(3 * j, 3 * j + 3)
        n = t if b == j else T
        assert torch.equal(got[b, h, :n], want[b, h, :n])
        if b == j:
            assert not torch.isfinite(got[b, h, t:]).any()
    assert not torch.isfinite(state[1, 1, 9]).any() and torch.isfinite(state[1, 1, :9]).all()


def test_long_prompts_over_several_runs():
    """A prompt that is split over tokens and heads: the runs' own sums carry
    the channel on, and nothing else."""
    B, hq, hkv, T = 1, 14, 2, 6000
    ld = [-0.0005, -0.03]
    q, k, v, s = _inputs(9, B, hq, hkv, T)
    want, wants = uc.linear_attend(q, k, v, ld, state=s)
    v[0, 1, 2500, 77] = INF
    got, state = uc.linear_attend(q, k, v, ld, state=s)
    assert torch.equal(got[:, :7], want[:, :7]) and torch.equal(state[:, 0], wants[:, 0])
    keep = torch.arange(128, device=got.device) != 77
    assert torch.equal(got[:, 7:, :, keep], want[:, 7:, :, keep])
    assert torch.equal(got[:, 7:, :2500], want[:, 7:, :2500])
    assert not torch.isfinite(got[:, 7:, 2500:, 77]).any() and not torch.isfinite(state[:, 1, :, 77]).any()
    assert torch.equal(state[:, 1, :, keep], wants[:, 1, :, keep])
