"""Layer norm and its gradients (float64, NumPy), from the definition.  TEST INFRASTRUCTURE ONLY - see oracle/__init__.py."""
from __future__ import annotations

import numpy as np


def forward(x, weight=None, bias=None, epsilon=1e-5):
    """(y, mean, rstd) of the rows of x: y = (x - mean) rstd w + b, rstd = (variance + epsilon)^(-1/2), divisor D."""
    x = np.asarray(x, np.float64)
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + epsilon)
    y = (x - mean[:, None]) * rstd[:, None]
    if weight is not None:
        y = y * np.asarray(weight, np.float64)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return y, mean, rstd


def backward(dy, x, mean, rstd, weight=None):
    """(dx, dweight, dbias) of sum(dy * y), with the mean and rstd of the forward pass."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    rstd = np.asarray(rstd, np.float64)[:, None]
    xhat = (x - np.asarray(mean, np.float64)[:, None]) * rstd
    g = dy if weight is None else dy * np.asarray(weight, np.float64)
    dx = rstd * (g - g.mean(axis=1, keepdims=True) - xhat * (g * xhat).mean(axis=1, keepdims=True))
    return dx, (dy * xhat).sum(axis=0), dy.sum(axis=0)
