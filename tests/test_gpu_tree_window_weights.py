"""GPU: softmax weights of trees behind a window are held in binary32, as without one, on every cache but the 4-bit one.

Bounds per element, for rows of bf16 calls over caches of bf16 and fp8 (A = the row's softmax average of |v|, S = its largest
scale * sum |q| |k|, n its keys, u = 2^-24): scores 2 D u S in a weight's exponent, numerator and denominator, an fp8 cache's scale
2 u S more; the sum of n weights n u, the sum of n values under weights that enter as three bf16 parts 3 n u; exponentials,
references, the merges of partial results and the division 32 u; the result's rounding 2^-8 of itself.  A weight rounded to bf16
would add up to 2^-8 A."""
import numpy as np
import pytest

from oracle import window as OW
from paper_2604_09731_amd import binding as B
from tests.test_gpu_tree_window import Case, U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return B.SmartTree(0)


def _check(c, out, lse, nodes):
    f = lambda x: x.double().cpu().numpy()
    got, got_lse, q, kt, vt, words = f(out), f(lse), f(c.q), f(c.kt), f(c.vt), c.mask.cpu().numpy()
    D = q.shape[2]
    for b in range(len(c.lens)):
        lo, hi = int(c.h_cu[b]), int(c.h_cu[b + 1])
        kp, vp = c.prefix(b)
        for i in sorted(nodes & set(range(lo, hi))):
            rows = OW.node_rows(q[i], kt[lo:hi], vt[lo:hi], OW.line_of(words[i], hi - lo), kp, vp, c.window, c.sinks, c.scale)
            for h, (ref, ref_lse, A, S, n) in enumerate(rows):
                u = ((2 * D + 2) * S + 4 * n + 32) * U
                err, tol = np.abs(got[i, h] - ref), u * A + 2.0 ** -8 * np.abs(ref)
                assert (err <= tol).all(), (b, i - lo, h, np.max(err / np.maximum(tol, 1e-300)))
                assert abs(got_lse[i, h] - ref_lse) <= u + 2 * U * abs(ref_lse), (b, i - lo, h)


@pytest.mark.parametrize("cache,layout", [("same", "interleaved"), ("same", "plain"), ("fp8", "interleaved"), ("fp8", "plain")])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,sizes,window,sinks", [
    ([0, 1, 30, 57, 130, 200], [3, 1, 4, 12, 9, 2], 9, 2),          # a workgroup a segment
    ([3001, 1500, 2222], [5, 20, 1], 1500, 13)])                    # shares, joined by the finishing kernel
def test_weights_are_not_rounded(lib, cache, layout, D, lens, sizes, window, sinks):
    c = Case(lib, lens, sizes, window, sinks, D=D, cache=cache, layout=layout, seed=D + window)
    out, lse = c.run(lib)
    _check(c, out, lse, set(range(int(c.h_cu[-1]))))
