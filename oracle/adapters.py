"""Oracle of the low-rank adapters of many requests, in fp64 (NumPy)."""
from __future__ import annotations

import numpy as np


def add(y, x, a, b, ids, scales=None, ranks=None):
    """fp64 (result, bound of its sums): out[m] = y[m] + scale (x[m] a_i^T) b_i^T,
    i = ids[m], y[m] where i is no adapter.  The bound is scale (|x| |a_i|^T)
    |b_i|^T, which rounding errors of the inner sums are relative to."""
    out, bound = y.astype(np.float64).copy(), np.zeros(y.shape)
    n, R = a.shape[:2]
    for m, i in enumerate(ids):
        if not 0 <= i < n:
            continue
        r = R if ranks is None else min(max(int(ranks[i]), 0), R)
        s = 1.0 if scales is None else float(scales[i])
        A, B, v = a[i, :r].astype(np.float64), b[i][:, :r].astype(np.float64), x[m].astype(np.float64)
        out[m] += s * (B @ (A @ v))
        bound[m] = abs(s) * (np.abs(B) @ (np.abs(A) @ np.abs(v)))
    return out, bound
