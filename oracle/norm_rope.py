"""CPU oracle: root-mean-square norm of each head, then its rotation, in binary64.  TEST INFRASTRUCTURE ONLY.

    y = x / sqrt(mean(x^2) + eps) * weight;  the rotation of y as in oracle/rope.py
"""
from __future__ import annotations

import numpy as np

from oracle import rope as R


def norm_rope(x, weight, position, eps, base, rotary_dim, pairing):
    """x [N, H, D], weight [D] or None: the result, and per element the sum of |y| over what the rotation mixes (what error
    bounds are made of)."""
    x = np.asarray(x, np.float64)
    w = np.ones(x.shape[-1]) if weight is None else np.asarray(weight, np.float64)
    y = np.empty_like(x)
    for t in range(x.shape[0]):
        for h in range(x.shape[1]):
            y[t, h] = x[t, h] / np.sqrt((x[t, h] * x[t, h]).sum() / x.shape[2] + eps) * w
    half, mixed = rotary_dim // 2, np.abs(y)
    for i in range(half):
        a, b = (i, i + half) if pairing == R.HALF_SPLIT else (2 * i, 2 * i + 1)
        both = np.abs(y[..., a]) + np.abs(y[..., b])
        mixed[..., a] = mixed[..., b] = both
    return R.rope(y, position, base, rotary_dim, pairing), mixed
