"""AdamW and its moments in 8 bits (float64, NumPy), from the definitions.  TEST INFRASTRUCTURE ONLY - see oracle/__init__.py."""
from __future__ import annotations

import numpy as np

BLOCK = 256
HALF = 0.5            # the share of a step that rounds to nearest


def step(p, g, m, v, t, lr, beta1=0.9, beta2=0.999, epsilon=1e-8, decay=0.0, scale=1.0):
    """(p, m, v) behind step t = 1, 2, ..."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    g = g * scale
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    p = p * (1.0 - lr * decay) - lr * (m / (1.0 - beta1 ** t)) / (np.sqrt(v / (1.0 - beta2 ** t)) + epsilon)
    return p, m, v


def share(n, t, start=0):
    """The share of a code's step that is added to elements start, start + 1, ... at step t."""
    i = np.arange(start, start + n, dtype=np.uint64)
    u = (i * np.uint64(0x9E3779B1) + np.uint64(t * 0x6A09E667 % 2 ** 32)) % np.uint64(2 ** 32)
    return (u >> np.uint64(12)).astype(np.float64) / 2.0 ** 20


def _exponent(a, lowest, highest):
    """The least E, not below `lowest`, with 1.875 2^E >= every finite number of the block; `highest` where that is highest + 1: the largest
    moments of fp32 are held as the largest code that stands for a number of fp32."""
    top = np.max(np.where(np.isfinite(a), a, 0.0), initial=0.0)
    if top == 0.0:
        return lowest
    f, e = np.frexp(top)
    E = max(int(e) - 1 if 2.0 * f <= 1.875 else int(e), lowest)
    return highest if E == highest + 1 else E


def _grid(a, shares):
    """Rounded down behind `shares` of a step, in eighths of the binade."""
    with np.errstate(invalid="ignore"):
        _, e = np.frexp(np.where(np.isfinite(a), a, 0.0))
        unit = np.exp2(e - 4.0)
        return np.floor(a / unit + shares) * unit


def coded_m(m, shares=HALF, top_of=None):
    """The values that the codes of one block of m stand for.  `top_of`: the numbers that set the exponent, if others."""
    m = np.asarray(m, np.float64)
    a = np.abs(m)
    E = _exponent(a if top_of is None else np.abs(top_of), 16 - 127, 127)
    least = 1.125 * 2.0 ** (E - 15)
    held = np.clip(_grid(a, shares), least, 1.875 * 2.0 ** E)
    held = np.where(a < least, np.where(a > shares * least, least, 0.0), held)
    return np.where(np.isfinite(m), np.sign(m) * held, np.nan)


def coded_v(v, shares=HALF, top_of=None):
    """The values that the codes of one block of v stand for: v is held by its root."""
    with np.errstate(invalid="ignore"):
        r = np.sqrt(np.asarray(v, np.float64))
        E = _exponent(r if top_of is None else np.sqrt(top_of), 32 - 127, 63)
    held = np.clip(_grid(r, shares), 1.25 * 2.0 ** (E - 31), 1.875 * 2.0 ** E)
    return np.where(np.isfinite(r), np.where(r > 0.0, held, 0.0) ** 2, np.nan)


def coded(which, a, t=None):
    """A flat array of blocks, coded at step t (None: to nearest)."""
    a = np.asarray(a, np.float64)
    out = np.empty_like(a)
    for at in range(0, len(a), BLOCK):
        out[at:at + BLOCK] = which(a[at:at + BLOCK], HALF if t is None else share(BLOCK, t, at))
    return out
