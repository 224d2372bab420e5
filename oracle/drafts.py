"""Verification of drafted tokens against the target's probabilities, in fp64.

Parity: pinned by hand-worked cases (tests/test_oracle_window.py). The paper has
no counterpart.
"""
from __future__ import annotations

import numpy as np


def log_softmax(x, temperature):
    x = np.asarray(x, np.float64) / temperature
    top = x.max(axis=-1, keepdims=True)
    return x - (top + np.log(np.exp(x - top).sum(axis=-1, keepdims=True)))


def verify(target, tokens, u=None, noise=None, draft=None, n_draft=None, temperature=1.0):
    """-> (accepted [B], tokens [B, T + 1], logprob [B, T + 1], margin [B]).

    margin: by what share of itself a probability or a weight may be off before a
    decision changes: of a draft |log(u q / p)|, of the next token the distance of
    the two best weights over what p + q at them may carry into it."""
    target = np.asarray(target, np.float64)
    B, T1, V = target.shape
    T = T1 - 1
    n = np.full(B, T) if n_draft is None else np.asarray(n_draft)
    lp = log_softmax(target, temperature or 1.0)
    lq = None if draft is None or temperature == 0 else log_softmax(draft, temperature)
    accepted, margin = np.zeros(B, np.int64), np.full(B, np.inf)
    out, logprob = np.full((B, T1), -1, np.int64), np.zeros((B, T1))
    for b in range(B):
        a = 0
        while a < n[b]:
            d = int(tokens[b, a])
            if temperature == 0:
                good = d == int(np.argmax(target[b, a]))
            else:
                good = False
                if 0 <= d < V:
                    p, q = np.exp(lp[b, a, d]), 1.0 if lq is None else np.exp(lq[b, a, d])
                    good = u[b, a] * q < p
                    if p > 0 and u[b, a] * q > 0:
                        margin[b] = min(margin[b], abs(np.log(u[b, a]) + np.log(q) - np.log(p)))
            if not good:
                break
            a += 1
        if temperature == 0:
            last = int(np.argmax(target[b, a]))
        else:
            p = np.exp(lp[b, a])
            q = np.zeros(V)
            if a < n[b]:
                if lq is not None:
                    q = np.exp(lq[b, a])
                elif 0 <= tokens[b, a] < V:
                    q[tokens[b, a]] = 1.0
            w = np.maximum(p - q, 0.0) / noise[b]
            last = int(np.argmax(w))
            err = (p + q) / noise[b]          # what a relative error of 1 would do
            others = np.delete(np.arange(V), last)
            if len(others):
                gap = (w[last] - w[others]) / (err[last] + err[others] + 1e-300)
                margin[b] = min(margin[b], gap.min())
        accepted[b] = a
        out[b, :a], out[b, a] = tokens[b, :a], last
        logprob[b, :a + 1] = lp[b, np.arange(a + 1), out[b, :a + 1]]
    return accepted, out, logprob, margin
