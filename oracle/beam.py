"""Oracle of the beam search's selection and of the reordering of states
(NumPy, fp64)."""
from __future__ import annotations

import numpy as np


def scores_of(logits: np.ndarray, scores: np.ndarray, finished=None, end_token=-1) -> np.ndarray:
    """fp64 [B, K, V]: the score of every continuation, -inf where it is none.
    logits [B * K, V], scores [B, K]."""
    B, K = scores.shape
    lg = np.asarray(logits, dtype=np.float64).reshape(B, K, -1)
    out = np.full(lg.shape, -np.inf)
    for b in range(B):
        for k in range(K):
            c = float(scores[b, k])
            if not np.isfinite(c):
                continue
            if finished is not None and finished[b, k]:
                out[b, k, end_token] = c
                continue
            row = lg[b, k]
            m = row.max()
            if not np.isfinite(m) or np.isnan(row).any():   # nothing allowed, a NaN, or +inf
                continue
            d = row - m   # (m and the log apart: their sum would lose the log beside a large m)
            out[b, k] = c + (d - np.log(np.exp(d).sum()))
    return out


def select(logits, scores, n, finished=None, end_token=-1):
    """(scores fp64 [B, n], parents, tokens, ended): the n best, equal scores by
    beam, then token."""
    s = scores_of(logits, scores, finished, end_token)
    B, K, V = s.shape
    vals = np.full((B, n), -np.inf)
    parents = np.full((B, n), -1, dtype=np.int64)
    tokens = np.full((B, n), -1, dtype=np.int64)
    ended = np.zeros((B, n), dtype=bool)
    for b in range(B):
        flat = s[b].reshape(-1)
        order = np.lexsort((np.arange(flat.size), -flat))[:n]
        order = order[flat[order] > -np.inf]
        m = order.size
        vals[b, :m], parents[b, :m], tokens[b, :m] = flat[order], order // V, order % V
        ended[b, :m] = order % V == end_token
        if finished is not None:
            ended[b, :m] |= np.asarray(finished[b], dtype=bool)[order // V]
    return vals, parents, tokens, ended


def reorder(src: np.ndarray, dst: np.ndarray, parents, beams, lengths=None) -> np.ndarray:
    """The destination after the reordering: rows first, positions in
    dimension 1."""
    new, old = dst.copy(), src.copy()
    B, n = parents.shape
    for b in range(B):
        used = src.shape[1] if lengths is None else min(max(int(lengths[b]), 0), src.shape[1])
        for j in range(n):
            p = int(parents[b, j])
            if 0 <= p < beams:
                new[b * n + j, :used] = old[b * beams + p, :used]
    return new
