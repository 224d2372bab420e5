"""Linear attention with a decay for each KV head, from its recurrence in fp64:
S_t = gamma S_{t-1} + k_t v_t^T, o_t = S_t^T q_t / sqrt(d).

Parity: pinned against the explicit sum over earlier tokens
(tests/test_oracle_generation.py). The paper has no counterpart.
"""
from __future__ import annotations

import numpy as np


def linear_attend(q, k, v, log_decay, state=None, lengths=None):
    """q [B, Hq, T, d], k, v [B, Hkv, T, d] -> (o [B, Hq, T, d], state [B, Hkv,
    d, d], var [B, Hq, T, d], size [B, Hkv, d, d]). Outputs behind a sequence's
    length are zero. var: the sum of squares of the terms that o adds up, over
    tokens and over state channels (what independent relative roundings of
    those terms are weighed with); size: the state of the terms' magnitudes."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    B, hq, T, d = q.shape
    hkv = k.shape[1]
    g = hq // hkv
    gamma = np.exp(np.asarray(log_decay, np.float64))
    o = np.zeros_like(q)
    var = np.zeros_like(q)
    end = np.zeros((B, hkv, d, d))
    size = np.zeros_like(end)
    for b in range(B):
        n = T if lengths is None else int(lengths[b])
        for j in range(hkv):
            s = np.zeros((d, d)) if state is None else np.asarray(state[b, j], np.float64).copy()
            mag = np.abs(s)
            heads = slice(j * g, (j + 1) * g)
            for t in range(n):
                s = gamma[j] * s + np.outer(k[b, j, t], v[b, j, t])
                mag = gamma[j] * mag + np.abs(np.outer(k[b, j, t], v[b, j, t]))
                o[b, heads, t] = q[b, heads, t] @ s
                var[b, heads, t] = (q[b, heads, t] ** 2) @ (s ** 2)
            if n:
                i = np.arange(n)
                gap = i[:, None] - i[None, :]
                w = np.where(gap >= 0, gamma[j] ** np.maximum(gap, 0), 0.0)
                p = np.einsum("htc,sc->hts", q[b, heads, :n], k[b, j, :n]) * w
                var[b, heads, :n] += (p ** 2) @ (v[b, j, :n] ** 2)
            end[b, j], size[b, j] = s, mag
    return o / np.sqrt(d), end, var / d, size
