"""Cross-entropy of logits and its gradient (float64, NumPy), from the definition.  TEST INFRASTRUCTURE ONLY - see oracle/__init__.py."""
from __future__ import annotations

import numpy as np


def cross_entropy(logits, labels, scale=1.0):
    """(loss of each row, gradient of scale * sum(loss)); a row whose label is outside the classes has zeros."""
    x, labels = np.asarray(logits, np.float64), np.asarray(labels)
    N, V = x.shape
    there = (labels >= 0) & (labels < V)
    at = np.where(there, labels, 0)[:, None]
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        top = x.max(axis=1, keepdims=True)
        e = np.exp(x - top)
        own = np.take_along_axis(e, at, 1)
        np.put_along_axis(e, at, 0.0, 1)
        others = e.sum(axis=1, keepdims=True)
        gap = top - np.take_along_axis(x, at, 1)
        loss = np.where(gap == 0, np.log1p(others), np.log(others + own) + gap)[:, 0]
        d = e / (others + own)
        np.put_along_axis(d, at, -others / (others + own), 1)
    return np.where(there, loss, 0.0), np.where(there[:, None], scale * d, 0.0)
