"""Pins of the oracle's linear attention and beam selection (CPU)."""
import math

import numpy as np

from oracle import beams as obeams
from oracle import linear as olinear


def test_linear_attend_is_the_sum_over_earlier_tokens():
    rng = np.random.default_rng(0)
    B, hq, hkv, T, d = 2, 4, 2, 9, 5
    q, k, v = rng.normal(size=(B, hq, T, d)), rng.normal(size=(B, hkv, T, d)), rng.normal(size=(B, hkv, T, d))
    s0 = rng.normal(size=(B, hkv, d, d))
    ld = [-0.1, -2.0]
    o, s, var, size = olinear.linear_attend(q, k, v, ld, s0, [T, 4])
    for b, n in ((0, T), (1, 4)):
        for h in range(hq):
            j = h // 2
            for t in range(n):
                want = math.exp(ld[j] * (t + 1)) * (q[b, h, t] @ s0[b, j])
                for u in range(t + 1):
                    want = want + math.exp(ld[j] * (t - u)) * (q[b, h, t] @ k[b, j, u]) * v[b, j, u]
                np.testing.assert_allclose(o[b, h, t], want / math.sqrt(d), rtol=1e-12, atol=1e-12)
            assert not o[b, h, n:].any()
        for j in range(hkv):
            want = math.exp(ld[j] * n) * s0[b, j]
            for u in range(n):
                want = want + math.exp(ld[j] * (n - 1 - u)) * np.outer(k[b, j, u], v[b, j, u])
            np.testing.assert_allclose(s[b, j], want, rtol=1e-12, atol=1e-12)
    assert (size >= np.abs(s) - 1e-12).all() and (var >= 0).all()


def test_linear_attend_in_two_calls_is_one_call():
    rng = np.random.default_rng(1)
    q, k, v = (rng.normal(size=(1, h, 11, 4)) for h in (2, 1, 1))
    o, s, _, _ = olinear.linear_attend(q, k, v, [-0.3])
    o1, s1, _, _ = olinear.linear_attend(q[:, :, :7], k[:, :, :7], v[:, :, :7], [-0.3])
    o2, s2, _, _ = olinear.linear_attend(q[:, :, 7:], k[:, :, 7:], v[:, :, 7:], [-0.3], s1)
    np.testing.assert_allclose(np.concatenate([o1, o2], axis=2), o, rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(s2, s, rtol=1e-12, atol=1e-13)


def test_beam_select_by_hand():
    # softmax (1/2, 1/4, 1/4) and (1/8, 7/8, 0)
    x = np.log(np.array([[[0.5, 0.25, 0.25], [0.125, 0.875, 0.0 + 1e-300]]]))
    x[0, 1, 2] = -np.inf
    sc, parent, token, fin, _ = obeams.beam_select(x, [[0.0, math.log(0.5)]], 4, eos=1)
    assert parent.tolist() == [[0, 1, 0, 0]]         # 1/2, 7/16, 1/4, 1/4
    assert token.tolist() == [[0, 1, 1, 2]]          # equal scores: the lower token
    np.testing.assert_allclose(np.exp(sc), [[0.5, 0.4375, 0.25, 0.25]], rtol=1e-12)
    assert fin.tolist() == [[False, True, True, False]]


def test_beam_select_ties_dead_and_finished_beams():
    x = np.zeros((1, 3, 4))
    # equal everything: beams in order, tokens in order
    _, parent, token, _, _ = obeams.beam_select(x, [[-1.0, -1.0, -1.0]], 6)
    assert parent.tolist() == [[0, 0, 0, 0, 1, 1]] and token.tolist() == [[0, 1, 2, 3, 0, 1]]
    # beam 0 finished: one candidate at its own score; beam 1 not alive
    sc, parent, token, fin, _ = obeams.beam_select(x, [[-0.5, -np.inf, -1.0]], 6, [[True, False, False]], eos=3)
    assert parent[0, 0] == 0 and token[0, 0] == 3 and sc[0, 0] == -0.5 and fin[0, 0]
    assert parent[0, 1:5].tolist() == [2, 2, 2, 2] and np.isneginf(sc[0, 5]) and parent[0, 5] == 0


def test_source_of():
    assert obeams.source_of([[1, 0], [1, 1]], 2).tolist() == [1, 0, 3, 3]
    assert obeams.source_of([[0, 0, 0], [0, 0, 0]], 1).tolist() == [0, 0, 0, 1, 1, 1]
