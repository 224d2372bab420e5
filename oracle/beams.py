"""Beam selection and the reordering of sequences, in fp64 and plain indexing.

Parity: pinned by hand-worked cases (tests/test_oracle_generation.py). The
paper has no counterpart.
"""
from __future__ import annotations

import numpy as np


def beam_select(logits, scores, n, finished=None, eos=-1):
    """logits [B, K, V], scores [B, K] -> (scores, parent, token, finished, gap)
    [B, n]; by descending score, then ascending beam, descending logit,
    ascending token. gap[b]: the least distance of two neighbouring finite
    scores of different beams among the first n + 1 (what rounding may swap)."""
    x = np.array(logits, np.float64) + 0.0
    scores = np.asarray(scores, np.float64)
    B, K, V = x.shape
    if finished is not None:
        fin = np.asarray(finished, bool)
        x[fin] = -np.inf
        x[fin, eos] = 0.0
    top = x.max(axis=-1, keepdims=True)
    base = np.where(np.isfinite(top), top, 0.0)
    with np.errstate(divide="ignore"):
        lse = np.log(np.exp(x - base).sum(axis=-1, keepdims=True))
    with np.errstate(invalid="ignore"):
        c = np.where(np.isneginf(x), -np.inf, scores[..., None] + ((x - base) - lse))
    out = [np.zeros((B, n)), np.zeros((B, n), np.int64), np.zeros((B, n), np.int64), np.zeros((B, n), bool)]
    gap = np.full(B, np.inf)
    beam, token = (a.ravel() for a in np.meshgrid(np.arange(K), np.arange(V), indexing="ij"))
    for b in range(B):
        order = np.lexsort((token, -x[b].ravel(), beam, -c[b].ravel()))[:n + 1]
        best = c[b].ravel()[order]
        for i in range(len(order) - 1):
            if beam[order[i]] != beam[order[i + 1]] and np.isfinite(best[i + 1]):
                gap[b] = min(gap[b], best[i] - best[i + 1])
        order = order[:n]
        out[0][b], out[1][b], out[2][b] = c[b].ravel()[order], beam[order], token[order]
        out[3][b] = token[order] == eos
        if finished is not None:
            out[3][b] |= fin[b, beam[order]]
    return (*out, gap)


def source_of(parent, n_from):
    """parent [G, n_to] -> the source sequence of every target sequence."""
    parent = np.asarray(parent)
    return (np.arange(parent.shape[0])[:, None] * n_from + parent).ravel()
