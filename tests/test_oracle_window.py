"""Hand-worked cases of the oracle's rotary positions, windows and drafts (CPU)."""
import numpy as np
import pytest

from oracle import drafts, rotary, window


def test_rotary_quarter_turns():
    x = np.arange(1.0, 7.0).reshape(1, 1, 6)
    f = [np.pi / 2, np.pi]
    got = rotary.rotary(x, [1], f, interleaved=True, scale=2.0)
    np.testing.assert_allclose(got[0, 0], [-4, 2, -6, -8, 5, 6], atol=1e-12)   # (1, 2) -> (-2, 1), (3, 4) -> (-3, -4)
    got = rotary.rotary(x, [1], f)
    np.testing.assert_allclose(got[0, 0], [-3, -2, 1, -4, 5, 6], atol=1e-12)   # (1, 3) -> (-3, 1), (2, 4) -> (-2, -4)


def test_rotary_turns_back():
    x = np.random.default_rng(0).standard_normal((2, 3, 5, 8))
    p = np.array([[0, 1, 7, 2 ** 31 - 1, 5], [9, 9, 9, 9, 9]])
    y = rotary.rotary(rotary.rotary(x, p, [1.0, 0.3]), -p, [1.0, 0.3])
    np.testing.assert_allclose(y, x, atol=1e-9)


def test_rows_of_a_ring():
    assert [window.row_of(p, 2, 5) for p in range(10)] == [0, 1, 2, 3, 4, 2, 3, 4, 2, 3]
    assert window.held_tokens(7, 2, 5) == {0: 0, 1: 1, 2: 5, 3: 6, 4: 4}
    assert window.held_tokens(0, 2, 5) == {}


def test_append_keeps_the_last_of_a_row():
    k = np.arange(1.0, 7.0).reshape(1, 1, 6, 1)
    ck, cv = window.append(np.zeros((1, 1, 4, 1)), np.zeros((1, 1, 4, 1)), k, -k, [1], [6], 1)
    assert ck.ravel().tolist() == [0, 4, 5, 6] and cv.ravel().tolist() == [0, -4, -5, -6]   # tokens 1 .. 6 in rows 1 .. 3


def test_attend_sees_window_and_sinks():
    # equal keys: the output is the mean of what is seen; tokens 0 .. 5 in a ring of 3 behind one sink hold 0, 3, 4, 5
    v = np.zeros((1, 1, 4, 1))
    for p in range(6):
        v[0, 0, window.row_of(p, 1, 4)] = 10.0 ** p
    k = np.zeros((1, 1, 4, 1))
    out, lse, _, _ = window.attend(np.ones((1, 1, 3, 1)), k, v, [6], [2], 2, 1)
    # tokens 4 (sees 0, 3, 4) and 5 (0, 4, 5); the third row is no query
    np.testing.assert_allclose(out.ravel(), [(1 + 1e3 + 1e4) / 3, (1 + 1e4 + 1e5) / 3, 0])
    np.testing.assert_allclose(lse.ravel(), [np.log(3), np.log(3), -np.inf])


def test_attend_weights():
    q = np.array([2.0, 0, 0, 0]).reshape(1, 1, 1, 4)
    k = np.zeros((1, 1, 2, 4))
    k[0, 0, 1, 0] = np.log(3.0)
    v = np.array([1.0, 5.0]).reshape(1, 1, 2, 1) * np.ones(4)
    out, lse, _, _ = window.attend(q, k, v, [2], [1], 2, 0)
    np.testing.assert_allclose(out.ravel(), 4.0)            # (1 + 3 * 5) / 4
    np.testing.assert_allclose(lse.ravel(), np.log(4.0))


def test_drafts():
    p = np.log([[0.5, 0.3, 0.2], [0.1, 0.6, 0.3]])[None]
    q = np.log([[0.2, 0.2, 0.6]])[None]
    e = np.array([[1.0, 1.0, 0.01]])
    # token 2: u q = 0.6 u < 0.2 while u < 1/3
    got = drafts.verify(p, np.array([[2]]), np.array([[0.3]]), e, q)
    assert got[0].tolist() == [1] and got[1].tolist() == [[2, 2]]       # w / e = 0.1, 0.6, 30
    np.testing.assert_allclose(got[2], np.log([[0.2, 0.3]]))
    got = drafts.verify(p, np.array([[2]]), np.array([[0.4]]), e, q)
    assert got[0].tolist() == [0] and got[1].tolist() == [[0, -1]]      # w = 0.3, 0.1, 0
    np.testing.assert_allclose(got[2], [[np.log(0.5), 0]])
    got = drafts.verify(p, np.array([[2]]), np.array([[0.4]]), e)       # a certain draft: token 2 is out
    assert got[0].tolist() == [0] and got[1].tolist() == [[0, -1]]
    got = drafts.verify(p, np.array([[2]]), np.array([[0.4]]), e, q, n_draft=[0])
    assert got[0].tolist() == [0] and got[1].tolist() == [[2, -1]]      # p_0 / e = 0.5, 0.3, 20
    got = drafts.verify(p, np.array([[0]]), temperature=0)
    assert got[0].tolist() == [1] and got[1].tolist() == [[0, 1]]
    got = drafts.verify(p, np.array([[1]]), temperature=0)
    assert got[0].tolist() == [0] and got[1].tolist() == [[0, -1]]


def test_drafts_leave_the_targets_distribution():
    """Over uniform u and exponential noise the first token is distributed as p."""
    rng = np.random.default_rng(1)
    p, q = np.array([0.5, 0.3, 0.2]), np.array([0.2, 0.2, 0.6])
    n = 20000
    tokens = rng.choice(3, size=(n, 1), p=q)
    got = drafts.verify(np.broadcast_to(np.log(p), (n, 2, 3)), tokens, rng.random((n, 1)), rng.exponential(size=(n, 3)),
                        np.broadcast_to(np.log(q), (n, 1, 3)))
    share = np.bincount(got[1][:, 0], minlength=3) / n
    assert np.abs(share - p).max() < 5 * 0.5 / np.sqrt(n)


def test_drafts_margin():
    p = np.log([[0.5, 0.5]])[None].repeat(2, axis=1)
    got = drafts.verify(p, np.array([[0]]), np.array([[0.5 * (1 - 1e-6)]]), np.ones((1, 2)))
    assert got[3][0] == pytest.approx(0.0)                   # two equal weights
    got = drafts.verify(p, np.array([[0]]), np.array([[0.5 * (1 - 1e-6)]]), np.array([[1.0, 9.0]]))
    assert got[3][0] == pytest.approx(1e-6, rel=1e-3)
