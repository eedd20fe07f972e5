"""CPU oracle: tree attention through a sliding window, in binary64.  TEST INFRASTRUCTURE ONLY.

Row by row over the keys that a node sees, so that nothing else enters it: with `line` the node's ancestors and itself from the root
down, positions are length + 0, 1, .. along it, and a key at position x is seen from position p if p - x < window or x < sinks.
"""
from __future__ import annotations

import numpy as np

from oracle import prompt as P


def seen_tokens(length, position, window, sinks):
    return [t for t in range(length) if position - t < window or t < sinks]


def line_of(words, n):
    """The set bits of a node's two mask words, of a tree of n nodes."""
    bits = (int(words[0]) & (2 ** 64 - 1)) | ((int(words[1]) & (2 ** 64 - 1)) << 64)
    return [j for j in range(n) if (bits >> j) & 1]


def node_rows(q, k_tree, v_tree, line, k_prefix, v_prefix, window, sinks, scale):
    """q [Hq, D] of one node; k_tree, v_tree [n, H, D]; k_prefix, v_prefix [length, H, D] float64.  Per head: output, log-sum-exp,
    average |v|, largest sum |q| |k|, number of keys."""
    length, G = len(k_prefix), q.shape[0] // k_tree.shape[1]
    position = length + max(len(line) - 1, 0)
    tokens = seen_tokens(length, position, window, sinks)
    nodes = [j for d, j in enumerate(line) if position - (length + d) < window or length + d < sinks]
    out = []
    for h in range(q.shape[0]):
        k = np.concatenate([k_prefix[tokens, h // G], k_tree[nodes, h // G]])
        v = np.concatenate([v_prefix[tokens, h // G], v_tree[nodes, h // G]])
        if not len(k):
            out.append((np.zeros(q.shape[1]), -np.inf, np.zeros(q.shape[1]), 0.0, 0))
        else:
            out.append((*P.prompt_row(q[h], k, v, scale), len(k)))
    return out
