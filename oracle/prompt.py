"""CPU oracle: causal attention of packed prompts, in binary64.  TEST INFRASTRUCTURE ONLY.

    out[t, h] = sum_{u <= t, same prompt} softmax_u(scale <q[t, h], k[u, h // G]>) v[u, h // G]

written row by row over the row's own keys, so that nothing else enters it.  With a window the keys are those u <= t with
t - u < window or u < sinks.
"""
from __future__ import annotations

import numpy as np


def seen(t, window, sinks):
    """The tokens that token t of a prompt sees, ascending."""
    return [u for u in range(t + 1) if window is None or t - u < window or u < sinks]


def prompt_attention(q, k, v, cu, scale, window=None, sinks=0):
    """q [T, Hq, D], k, v [T, Hkv, D] float64; returns out, lse [T, Hq], and per element the softmax average of |v| and per
    row the largest sum |q| |k| (what error bounds are made of).  Rows of no prompt stay NaN."""
    T, Hq, D = q.shape
    G = Hq // k.shape[1]
    out, mean_abs = np.full((T, Hq, D), np.nan), np.full((T, Hq, D), np.nan)
    lse, size = np.full((T, Hq), np.nan), np.full((T, Hq), np.nan)
    for lo, hi in zip(cu[:-1], cu[1:]):
        for t in range(lo, hi):
            for h in range(Hq):
                own = slice(lo, t + 1) if window is None else lo + np.array(seen(t - lo, window, sinks))
                out[t, h], lse[t, h], mean_abs[t, h], size[t, h] = prompt_row(q[t, h], k[own, h // G], v[own, h // G], scale)
    return out, lse, mean_abs, size


def prompt_row(q, keys, values, scale):
    """One row over its own keys: its output, log-sum-exp, average of |v| and largest sum |q| |k|."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = scale * (keys @ q)
        m = s.max()
        p = np.exp(s - m)
        w = p / p.sum()
        return w @ values, m + np.log(p.sum()), w @ np.abs(values), scale * (np.abs(keys) @ np.abs(q)).max()
