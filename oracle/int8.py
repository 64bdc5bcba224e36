"""Oracle of the 8-bit integer product and of the rounding that feeds it, in
fp64 and whole numbers (NumPy)."""
from __future__ import annotations

import numpy as np

TINY = 2.0 ** -126   # smallest scale of a row


def quantize(x: np.ndarray):
    """Rows of x (any float type, exact in fp64) -> (codes int8, scales fp32):
    scale = max(|x| / 127 of the row's largest, 2^-126) in fp32, code = the
    integer nearest to x / scale, halves to even.  Quotients of 24-bit numbers
    that are not halves differ from one by more than 2^-26, so fp64 decides
    them.  A row that is not finite: scale NaN, codes 0."""
    x = np.asarray(x, dtype=np.float64)
    bad = ~np.isfinite(x).all(axis=1)
    y = np.where(bad[:, None], 0.0, x)
    s = np.maximum((np.abs(y).max(axis=1) / 127.0).astype(np.float32), np.float32(TINY))
    q = np.rint(y / s.astype(np.float64)[:, None]).astype(np.int8)
    return q, np.where(bad, np.float32(np.nan), s)


def matmul(a, sa, b, sb, bias=None):
    """(fp64 result, fp64 product before the bias): the sums are whole numbers
    far below 2^53, exact in fp64 in any order."""
    acc = a.astype(np.float64) @ b.astype(np.float64).T
    p = acc * sa.astype(np.float64)[:, None] * sb.astype(np.float64)
    return (p if bias is None else p + bias.astype(np.float64)), p
