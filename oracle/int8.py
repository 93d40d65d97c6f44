"""Rows of 8-bit integers with a float32 scale each, and their products, plain float64 NumPy (oracle: test
infrastructure only).

* scale of a row: max|x| / 127 rounded to float32, at least 2^-126; q: the whole number nearest to x / scale, ties to
  even. x and scale have 24 significant bits, so that a float64 quotient lies on the right side of every border.
* a row with a NaN or an infinity: scale NaN, zeros.
"""
from __future__ import annotations

import numpy as np


def quantise(x: np.ndarray):
    """(q int8 [R][K], scale float32 [R])."""
    x = np.asarray(x, np.float64)
    good = np.isfinite(x).all(axis=1)
    x = np.where(good[:, None], x, 0.0)
    s = np.maximum((np.abs(x).max(axis=1) / 127.0).astype(np.float32), np.float32(2.0 ** -126))
    q = np.rint(x / s[:, None].astype(np.float64))
    assert np.all(np.abs(q) <= 127)
    return q.astype(np.int8), np.where(good, s, np.float32(np.nan))


def linear(q: np.ndarray, scale: np.ndarray, wq: np.ndarray, w_scale: np.ndarray, bias=None) -> np.ndarray:
    """scale[m] w_scale[n] sum_k q[m][k] wq[n][k] + bias[n]; the sums are exact (whole numbers below 2^53)."""
    s = q.astype(np.float64) @ wq.astype(np.float64).T
    v = scale.astype(np.float64)[:, None] * (w_scale.astype(np.float64) * s)
    return v if bias is None else v + bias.astype(np.float64)
