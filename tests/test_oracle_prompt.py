"""The prompt attention oracle against closed forms."""
import numpy as np

from oracle import prompt as P


def test_closed_forms():
    rng = np.random.default_rng(0)
    cu = [2, 5, 5, 9]
    q, k, v = rng.standard_normal((10, 4, 8)), rng.standard_normal((10, 2, 8)), rng.standard_normal((10, 2, 8))
    out, lse, _, _ = P.prompt_attention(q, k, v, cu, 0.5)
    assert np.isnan(out[:2]).all() and np.isnan(out[9:]).all() and np.isfinite(out[2:9]).all()
    for first in (2, 5):                                    # a first token sees itself only
        for h in range(4):
            assert np.allclose(out[first, h], v[first, h // 2], atol=1e-15)
            assert np.isclose(lse[first, h], 0.5 * q[first, h] @ k[first, h // 2])
    # equal keys: plain means of the values so far
    out, lse, _, _ = P.prompt_attention(q, np.ones_like(k), v, [0, 10], 0.5)
    assert np.allclose(out[:, 1], np.cumsum(v[:, 0], 0) / np.arange(1, 11)[:, None])
    assert np.allclose(lse[:, 1], 0.5 * q[:, 1].sum(1) + np.log(np.arange(1, 11)))


def test_later_tokens_never_enter():
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal((6, 1, 4)) for _ in range(3))
    ref = P.prompt_attention(q, k, v, [0, 6], 1.0)[0]
    k[4:], v[4:] = np.inf, np.nan
    assert np.array_equal(P.prompt_attention(q, k, v, [0, 6], 1.0)[0][:4], ref[:4])
