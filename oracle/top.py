"""Oracle selection of the largest logits of each row, and the log-sum-exp.

TEST INFRASTRUCTURE ONLY (see the package docstring).

Order: value descending, then column ascending; NaN above all numbers, -0 as 0.
"""
from __future__ import annotations

import numpy as np


def top(z, k):
    """z [rows, vocab] float64 -> (columns [rows, k], values [rows, k])."""
    ids = np.empty((len(z), k), np.int32)
    for r, row in enumerate(z):
        nan = np.isnan(row)
        key = np.where(nan, 0.0, row)
        # sorted by the last key first: not NaN, then value, then column (stable)
        ids[r] = np.lexsort((np.arange(len(row)), -key, ~nan))[:k]
    return ids, np.take_along_axis(z, ids, 1)


def lse(z, scale=1.0):
    y = z * scale
    m = y.max(1)
    with np.errstate(all="ignore"):
        ref = np.where(np.isfinite(m), m, 0.0)
        return ref + np.log(np.exp(y - ref[:, None]).sum(1))
