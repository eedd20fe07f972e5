"""CPU oracle: causal attention of packed prompts, in binary64.  TEST INFRASTRUCTURE ONLY.

    out[t, h] = sum_{u <= t, same prompt} softmax_u(scale <q[t, h], k[u, h // G]>) v[u, h // G]

written row by row over the row's own keys, so that nothing else enters it.
"""
from __future__ import annotations

import numpy as np


def prompt_attention(q, k, v, cu, scale):
    """q [T, Hq, D], k, v [T, Hkv, D] float64; returns out, lse [T, Hq], and per element the softmax average of |v| and per
    row the largest sum |q| |k| (what error bounds are made of).  Rows of no prompt stay NaN."""
    T, Hq, D = q.shape
    G = Hq // k.shape[1]
    out, mean_abs = np.full((T, Hq, D), np.nan), np.full((T, Hq, D), np.nan)
    lse, size = np.full((T, Hq), np.nan), np.full((T, Hq), np.nan)
    with np.errstate(invalid="ignore", over="ignore"):
        for lo, hi in zip(cu[:-1], cu[1:]):
            for h in range(Hq):
                g = h // G
                for t in range(lo, hi):
                    keys, values = k[lo:t + 1, g], v[lo:t + 1, g]
                    s = scale * (keys @ q[t, h])
                    m = s.max()
                    p = np.exp(s - m)
                    w = p / p.sum()
                    out[t, h] = w @ values
                    mean_abs[t, h] = w @ np.abs(values)
                    lse[t, h] = m + np.log(p.sum())
                    size[t, h] = scale * (np.abs(keys) @ np.abs(q[t, h])).max()
    return out, lse, mean_abs, size
