"""Norm of many tensors as one vector and the factor of clipping (float64, NumPy).  TEST INFRASTRUCTURE ONLY - see oracle/__init__.py."""
from __future__ import annotations

import numpy as np


def norm_and_factor(tensors, max_norm):
    """sqrt of the sum of all squares, and max_norm / norm where the norm is above max_norm, else 1 (a NaN stays one)."""
    norm = float(np.sqrt(sum(float(np.sum(np.square(np.asarray(t, np.float64)))) for t in tensors if t is not None)))
    if np.isnan(norm):
        return norm, norm
    return norm, (max_norm / norm if norm > max_norm else 1.0)
