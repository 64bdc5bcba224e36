"""Oracle of the root-mean-square norm with the residual's addition and the
rounding of its rows to 8 bits, in fp64 (NumPy)."""
from __future__ import annotations

import numpy as np

from . import int8


def rms_norm(x, weight, eps, residual=None, offset=0.0):
    """fp32 arrays holding the inputs' values -> (s, t, n, codes, u): s = x +
    residual and t = s (offset + weight) rounded to fp32, n = sqrt(mean s^2 + eps)
    in fp64 [M], codes int8 and step u of t (its scale before 1 / n; NaN where t
    is not finite)."""
    with np.errstate(over="ignore", invalid="ignore"):
        x = np.asarray(x, np.float32)
        s = x if residual is None else x + np.asarray(residual, np.float32)
        t = s * (np.float32(offset) + np.asarray(weight, np.float32))
        n = np.sqrt((s.astype(np.float64) ** 2).mean(axis=1) + eps)
    codes, u = int8.quantize(t)
    return s, t, n, codes, u
