"""The norm-and-rotation oracle against closed forms."""
import numpy as np

from oracle import norm_rope as N
from oracle import rope as R


def test_norms_lengths_and_weights():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((4, 3, 16)) * 7
    for pairing in (R.HALF_SPLIT, R.INTERLEAVED):
        y, mixed = N.norm_rope(x, None, [0, 5, 900, 70000], 1e-12, 100.0, 16, pairing)
        assert np.allclose((y ** 2).mean(-1), 1.0)                   # a rotation keeps lengths
        assert (np.abs(y) <= mixed + 1e-12).all()
        assert np.allclose(N.norm_rope(x * 3, None, [0, 5, 900, 70000], 1e-12, 100.0, 16, pairing)[0], y)
    w = rng.standard_normal(16)
    plain = N.norm_rope(x, w, [0] * 4, 0.5, 100.0, 8, R.HALF_SPLIT)[0]
    assert np.allclose(plain, x / np.sqrt((x ** 2).mean(-1, keepdims=True) + 0.5) * w)
    assert np.array_equal(N.norm_rope(x, w, [3] * 4, 0.5, 100.0, 8, R.HALF_SPLIT)[0][..., 8:], plain[..., 8:])
    assert not N.norm_rope(np.zeros((1, 1, 4)), None, [9], 1e-6, 10.0, 4, R.HALF_SPLIT)[0].any()
