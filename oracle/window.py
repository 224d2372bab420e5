"""The cache of a layer with a sliding window and first tokens, and attention
over it, in fp64, token by token.

Parity: pinned by hand-worked cases (tests/test_oracle_window.py). The paper has
no counterpart.
"""
from __future__ import annotations

import numpy as np


def row_of(p, n_sink, n_rows):
    """The cache's row of token p."""
    return p if p < n_sink else n_sink + (p - n_sink) % (n_rows - n_sink)


def held_tokens(length, n_sink, n_rows):
    """{row: token} after ``length`` tokens came one after the other."""
    held = {}
    for p in range(length):
        held[row_of(p, n_sink, n_rows)] = p
    return held


def append(cache_k, cache_v, k, v, held, n_new, n_sink):
    """New tokens k, v [B, H, T, D] into copies of the caches [B, H, rows, D]."""
    ck, cv = np.array(cache_k), np.array(cache_v)
    for b in range(ck.shape[0]):
        for t in range(n_new[b]):
            r = row_of(held[b] + t, n_sink, ck.shape[2])
            ck[b, :, r], cv[b, :, r] = k[b, :, t], v[b, :, t]
    return ck, cv


def attend(q, cache_k, cache_v, lengths, n_query, window, n_sink):
    """q [B, Hq, T, D] -> (out, lse, spread, reach): spread [B, Hq, T, D] = sum p
    |v| and reach [B, Hq, T] = the largest sum |q k| / sqrt(D), what errors of p
    and of the logits are measured by. Rows that see nothing: 0 and -inf."""
    q = np.asarray(q, np.float64)
    B, hq, T, D = q.shape
    hkv, rows = cache_k.shape[1], cache_k.shape[2]
    grp = hq // hkv
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    lse, reach = np.full((B, hq, T), -np.inf), np.zeros((B, hq, T))
    for b in range(B):
        held = held_tokens(int(lengths[b]), n_sink, rows)
        where = sorted((p, r) for r, p in held.items())
        token = np.array([p for p, _ in where], np.int64)
        at = np.array([r for _, r in where], np.int64)
        for t in range(int(n_query[b])):
            p = int(lengths[b]) - int(n_query[b]) + t
            see = (token <= p) & ((p - token < window) | (token < n_sink))
            if not see.any():
                continue
            for j in range(hkv):
                k = np.asarray(cache_k[b, j][at[see]], np.float64)
                v = np.asarray(cache_v[b, j][at[see]], np.float64)
                h = slice(j * grp, (j + 1) * grp)
                x = q[b, h, t] @ k.T / np.sqrt(D)
                top = x.max(axis=-1, keepdims=True)
                e = np.exp(x - top)
                total = e.sum(axis=-1, keepdims=True)
                out[b, h, t] = e / total @ v
                spread[b, h, t] = e / total @ np.abs(v)
                lse[b, h, t] = (np.log(total) + top)[..., 0]
                reach[b, h, t] = (np.abs(q[b, h, t]) @ np.abs(k).T).max(axis=-1) / np.sqrt(D)
    return out, lse, spread, reach
