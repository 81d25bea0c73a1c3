"""Root-mean-square norm with the residual's addition and its gradient, binary64, row by row.

TEST INFRASTRUCTURE ONLY.  READING: the residual stream is stored in its own type, so what is normalised is the rounded
sum; everything after that is binary64 here.  Pins: tests/test_oracle_norm.py.
"""
from __future__ import annotations

import numpy as np


def forward(h: np.ndarray, weight: np.ndarray, eps: float):
    """(rstd [rows], y) of rows h that are already rounded to the stream's type."""
    h, weight = h.astype(np.float64), weight.astype(np.float64)
    rstd = np.array([1.0 / np.sqrt(np.dot(r, r) / len(r) + eps) for r in h])
    return rstd, h * rstd[:, None] * weight


def backward(dy: np.ndarray, h: np.ndarray, weight: np.ndarray, rstd: np.ndarray, dres=None):
    """(dx, dw) from the forward pass's rstd."""
    dy, h, weight, rstd = (np.asarray(t, np.float64) for t in (dy, h, weight, rstd))
    dx, dw = np.zeros_like(h), np.zeros(h.shape[1])
    for i in range(h.shape[0]):
        n, g = h[i] * rstd[i], dy[i] * weight
        dx[i] = rstd[i] * (g - n * np.mean(g * n)) + (0.0 if dres is None else np.asarray(dres[i], np.float64))
        dw += dy[i] * n
    return dx, dw
