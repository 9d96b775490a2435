"""Lookup of table rows by tokens and the table's gradient (float64, NumPy), from the definition.  TEST INFRASTRUCTURE ONLY - see
oracle/__init__.py."""
from __future__ import annotations

import numpy as np


def forward(tokens, table, scale=1.0):
    """scale * table[token] for each token, zeros where it is outside the table."""
    table = np.asarray(table, np.float64)
    y = np.zeros((len(tokens), table.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < len(table):
            y[i] = scale * table[t]
    return y


def backward(dy, tokens, vocabulary, scale=1.0):
    """Gradient of sum(dy * forward) by the table."""
    dy, tokens = np.asarray(dy, np.float64), np.asarray(tokens)
    out = np.zeros((vocabulary, dy.shape[1]))
    named = (tokens >= 0) & (tokens < vocabulary)
    np.add.at(out, tokens[named], dy[named])
    return scale * out
