"""The window oracles against brute force over positions, and windows that hide nothing against the oracles without."""
import numpy as np

from oracle import prompt as P
from oracle import window as W


def test_prompts():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((9, 2, 4)), rng.standard_normal((9, 1, 4)), rng.standard_normal((9, 1, 4))
    full = P.prompt_attention(q, k, v, [0, 9], 0.5)
    for window, sinks in ((9, 0), (1, 9), (4, 5), (100, 100)):
        for x, y in zip(P.prompt_attention(q, k, v, [0, 9], 0.5, window, sinks), full):
            assert np.allclose(x, y)
    assert P.seen(7, 3, 2) == [0, 1, 5, 6, 7] and P.seen(2, 1, 0) == [2] and P.seen(3, 2, 3) == [0, 1, 2, 3]
    alone = P.prompt_attention(q, k, v, [0, 9], 0.5, 1, 0)[0]
    assert np.allclose(alone[:, 1], v[:, 0])


def test_a_chain_of_nodes_is_a_prompt():
    rng = np.random.default_rng(1)
    T, L = 14, 9
    q, k, v = rng.standard_normal((T, 2, 4)), rng.standard_normal((T, 2, 4)), rng.standard_normal((T, 2, 4))
    for window, sinks in ((1, 0), (3, 0), (4, 2), (7, 11), (50, 1)):
        out, lse, _, _ = P.prompt_attention(q, k, v, [0, T], 0.7, window, sinks)
        for i in range(T - L):
            rows = W.node_rows(q[L + i], k[L:], v[L:], list(range(i + 1)), k[:L], v[:L], window, sinks, 0.7)
            for h in range(2):
                assert np.allclose(rows[h][0], out[L + i, h]) and np.isclose(rows[h][1], lse[L + i, h])


def test_lines():
    assert W.line_of(np.array([0b1011, -1]), 3) == [0, 1] and W.line_of(np.array([-2 ** 63, 1]), 65) == [63, 64]
    out = W.node_rows(np.ones((1, 2)), np.ones((1, 1, 2)), np.ones((1, 1, 2)), [], np.ones((3, 1, 2)), np.ones((3, 1, 2)), 1, 0, 1.0)
    assert out[0][1] == -np.inf and out[0][4] == 0          # a node without a mask at position 3 sees nothing through a window of one
