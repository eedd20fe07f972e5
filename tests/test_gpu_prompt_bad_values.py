"""prompt_attention where values are infinite, NaN or near the end of the range: which rows they reach, and what such a call costs.

Bounds as in test_gpu_prompt_attention.py; a row that is evaluated again holds its weights in binary32, which they cover."""
import numpy as np
import pytest

from oracle import prompt as P
from paper_2604_09731_amd import binding as B
from tests.test_gpu_prompt_attention import U, _f64, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return B.SmartTree(0)


def _some_rows(out, q, k, v, lo, tokens, heads, scale, dtype):
    """Rows of the prompt that begins at `lo` against the oracle: finite where it is, infinite of the same sign or NaN where it is."""
    q, k, v, out = (_f64(x) for x in (q, k, v, out))
    D, G = q.shape[2], q.shape[1] // k.shape[1]
    for t in tokens:
        for h in heads:
            with np.errstate(invalid="ignore"):
                ref, _, A, S = P.prompt_row(q[t, h], k[lo:t + 1, h // G], v[lo:t + 1, h // G], scale)
            got, good = out[t, h], np.isfinite(ref)
            assert np.array_equal(np.isnan(got), np.isnan(ref)), (t, h)
            assert np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)]), (t, h)
            u = (2 * D * S + 2 * (t + 1 - lo) + 16) * U
            tol = u * A + (2 * 2.0 ** -8 * A + 2.0 ** -8 * np.abs(ref) if dtype == "bf16" else U * np.abs(ref))
            off = np.abs(got[good] - ref[good])
            assert (off <= tol[good]).all(), (t, h, (off / tol[good]).max())


@pytest.mark.parametrize("dtype,D,lens", [("bf16", 128, [300, 90]), ("bf16", 64, [1030]), ("f32", 64, [300, 90]), ("f32", 128, [260])])
@pytest.mark.parametrize("poison", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("at", [0, 16, 70, 89])
def test_a_bad_value_reaches_the_rows_that_see_it_and_their_head_dim_only(lib, dtype, D, lens, poison, at):
    """Some head dims of one token, and of another two tokens later (of the other sign)."""
    import torch
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    q, k, v = _inputs(int(cu[-1]), 6, 2, D, dtype, 41)
    clean = lib.prompt_attention(q, k, v, torch.from_numpy(cu).cuda(), D ** -0.5)
    lo = int(cu[-2])
    v[lo + at, 0, 5], v[lo + at, 1, D - 1], v[lo + at + 2 if at < 80 else lo, 0, [5, 9]] = poison, poison, -poison
    out = lib.prompt_attention(q, k, v, torch.from_numpy(cu).cuda(), D ** -0.5)
    if lo:
        assert torch.equal(out[:lo], clean[:lo])
    n = lens[-1]
    tokens = {0, at - 1, at, at + 1, at + 2, at + 3, at + 40, n - 1}
    _some_rows(out, q, k, v, lo, [lo + t for t in sorted(tokens) if 0 <= t < n], range(6), D ** -0.5, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_values_near_the_end_of_the_range(lib, dtype, D):
    """Values whose weighted sum stays inside binary32 as long as no weight exceeds 1, under scores that rise by less than the step in
    which the reference follows the maximum: 0 for the first 100 tokens, then 5."""
    import torch
    n = 512
    q, k, v = (torch.zeros((n, h, D), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda") for h in (2, 1, 1))
    q.fill_(1.0)
    k[100:] = 5.0 / D
    v.fill_(2.0 ** 118)
    out = lib.prompt_attention(q, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), 1.0)
    assert ((out.double() / 2.0 ** 118 - 1).abs() <= 2.0 ** -8).all()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_a_bad_value_of_the_first_token_costs_no_more_than_some_calls(lib, dtype, D):
    """Every row of the call sees it and comes out infinite there.  (Rows that are looked at one by one would take hundreds of
    times the call.)"""
    import torch
    n, Hq, Hkv = 3000, 16, 4
    q, k, v = _inputs(n, Hq, Hkv, D, dtype, 43)
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)

    def timed():
        lib.prompt_attention(q, k, v, cu, D ** -0.5, out=out)
        start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        lib.prompt_attention(q, k, v, cu, D ** -0.5, out=out)
        stop.record()
        torch.cuda.synchronize()
        return start.elapsed_time(stop)

    clean = min(timed() for _ in range(3))
    v[0, :, 7] = float("inf")
    slow = min(timed() for _ in range(3))
    print(f"{dtype} {D}: {clean * 1e3:.0f} us, with the infinity {slow * 1e3:.0f}")
    assert (out[:, :, 7] == float("inf")).all()
    _some_rows(out, q, k, v, 0, [0, 1, 777, n - 1], [0, Hq - 1], D ** -0.5, dtype)
    assert slow <= 40 * clean


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("at", [0, 40])
def test_rows_with_scores_that_are_no_numbers_have_no_log_sum_exp(lib, dtype, D, bad, at):
    """A NaN or an infinite score: the row is NaN, and its log-sum-exp too (not -infinity, which says that nothing has weight)."""
    import torch
    n = 150
    q, k, v = _inputs(n, 4, 2, D, dtype, 44)
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    clean, clean_lse = lib.prompt_attention(q, k, v, cu, D ** -0.5, want_lse=True)
    q[..., 3] = 1.0
    k[at, 1, 3] = bad                                   # of kv head 1: query heads 2 and 3
    q[90, 0, 7] = float("nan")
    out, lse = lib.prompt_attention(q, k, v, cu, D ** -0.5, want_lse=True)
    assert out[at:, 2:].isnan().all() and lse[at:, 2:].isnan().all()
    assert out[90, 0].isnan().all() and lse[90, 0].isnan()
    assert torch.isfinite(out[:at]).all() and torch.isfinite(lse[:at]).all()
    others = [t for t in range(n) if t != 90]
    assert torch.isfinite(out[others, :2]).all() and torch.isfinite(lse[others, :2]).all()
    assert torch.isfinite(clean).all() and torch.isfinite(clean_lse).all()
