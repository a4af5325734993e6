"""Matrices of 8-bit integers with a scale for each row, in numpy: from the definitions, quotients as fractions where they lie next to a half."""

from fractions import Fraction

import numpy as np


def quantize(x):
    """(integers, scales float64) of a float32 matrix: round(127 x / max|x|) of each row, ties to even; max|x| / 127."""
    x = np.asarray(x, np.float64)
    q = np.zeros(x.shape, np.int64)
    scales = np.zeros(x.shape[0])
    for i, row in enumerate(x):
        most = np.abs(row).max() if row.size else 0.0
        if not np.isfinite(most):
            scales[i] = np.nan
            continue
        scales[i] = most / 127
        if most == 0:
            continue
        up = 2.0 ** 200 if most < 1e-30 else 1.0
        t = 127 * (row * up) / (most * up)
        q[i] = np.rint(t)
        for j in np.nonzero(np.abs(np.abs(t - np.floor(t)) - 0.5) < 1e-9)[0]:
            q[i, j] = round(127 * Fraction(float(row[j])) / Fraction(float(most)))      # (Python rounds ties to even)
    return q, scales


def product(qa, sa, qb, sb, bias=None, relu=False):
    out = (qa.astype(np.int64) @ qb.astype(np.int64).T).astype(np.float64) * np.asarray(sa, np.float64)[:, None] * np.asarray(sb, np.float64)[None]
    if bias is not None:
        out = out + np.asarray(bias, np.float64)
    return np.where(out > 0, out, np.where(np.isnan(out), out, 0.0)) if relu else out
