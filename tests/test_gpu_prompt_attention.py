"""GPU parity of prompt_attention with the binary64 oracle.

Bounds per element, from what the kernel rounds (A = the row's softmax average of |v|, S = the row's largest
scale * sum |q| |k|, n its keys, u = 2^-24):
  a score is a binary32 sum of D products: off by at most D u S; it enters a weight's exponent, numerator and denominator;
  sums of n weights or weighted values: n u of A each; exponential, reference and division: 16 u;
  bf16: a weight is off by 2^-9 of itself at most once as a value and once in the sum that divides (2 2^-8 A bounds both), and
  the result is rounded to 8 bits (2^-8 of itself)."""
import numpy as np
import pytest

from oracle import prompt as P
from paper_2604_09731_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return B.SmartTree(0)


def _inputs(T, Hq, Hkv, D, dtype, seed, k_scale=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    return [(torch.randn((T, H, D), generator=g) * s).to(dt).cuda() for H, s in ((Hq, 1.0), (Hkv, k_scale), (Hkv, 1.0))]


def _f64(t):
    return t.double().cpu().numpy()


def _check(out, lse, q, k, v, cu, scale, dtype):
    D = q.shape[2]
    ref, ref_lse, A, S = P.prompt_attention(_f64(q), _f64(k), _f64(v), cu, scale)
    lens = np.full(q.shape[0], 1)
    for lo, hi in zip(cu[:-1], cu[1:]):
        lens[lo:hi] = np.arange(1, hi - lo + 1)
    own = np.zeros(q.shape[0], bool)
    own[cu[0]:cu[-1]] = True
    u = (2 * D * S + 2 * lens[:, None] + 16) * U
    tol = u[..., None] * A + (2 * 2.0 ** -8 * A + 2.0 ** -8 * np.abs(ref) if dtype == "bf16" else U * np.abs(ref))
    got = _f64(out)
    assert (np.abs(got - ref)[own] <= tol[own]).all(), np.nanmax((np.abs(got - ref) / tol)[own])
    if lse is not None:
        err = np.abs(lse.double().cpu().numpy() - ref_lse)
        assert (err[own] <= (u + 2 * U * np.abs(ref_lse))[own]).all(), np.nanmax((err / u)[own])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (7, 1)])
@pytest.mark.parametrize("lens", [[1], [37], [0, 5, 0, 64, 33, 1, 0], [129, 31, 32, 255]])
def test_against_the_oracle(lib, dtype, D, Hq, Hkv, lens):
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    import torch
    q, k, v = _inputs(int(cu[-1]), Hq, Hkv, D, dtype, 3 + sum(lens))
    out, lse = lib.prompt_attention(q, k, v, torch.from_numpy(cu).cuda(), D ** -0.5, want_lse=True)
    _check(out, lse, q, k, v, cu, D ** -0.5, dtype)
    bare = lib.prompt_attention(q, k, v, torch.from_numpy(cu).cuda(), D ** -0.5)
    assert torch.equal(bare, out)


@pytest.mark.parametrize("dtype,D,lens", [("bf16", 128, [700, 3, 450]), ("bf16", 64, [1030]), ("f32", 128, [600]), ("f32", 64, [513, 200])])
def test_several_row_tiles(lib, dtype, D, lens):
    import torch
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    q, k, v = _inputs(int(cu[-1]), 6, 2, D, dtype, 77)
    out, lse = lib.prompt_attention(q, k, v, torch.from_numpy(cu).cuda(), D ** -0.5, want_lse=True)
    _check(out, lse, q, k, v, cu, D ** -0.5, dtype)


@pytest.mark.parametrize("D,Hq,Hkv,lens", [(128, 28, 4, [1500, 2, 700]), (64, 32, 8, [1500, 2, 700]),
                                           (128, 64, 8, [3000, 1, 0, 1200, 77]), (64, 64, 8, [3000, 1, 0, 1200, 77])])
@pytest.mark.parametrize("lse", [False, True])
def test_large_calls_by_some_of_their_rows(lib, D, Hq, Hkv, lens, lse):
    """Calls of enough rows for the taller row tiles; the oracle on the first, last and random rows of every prompt."""
    import torch
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    q, k, v = _inputs(int(cu[-1]), Hq, Hkv, D, "bf16", 31)
    got = lib.prompt_attention(q, k, v, torch.from_numpy(cu).cuda(), D ** -0.5, want_lse=lse)
    out, got_lse = (_f64(got[0]), _f64(got[1])) if lse else (_f64(got), None)
    assert np.isfinite(out).all()
    q, k, v = _f64(q), _f64(k), _f64(v)
    rng = np.random.default_rng(0)
    for lo, hi in zip(cu[:-1], cu[1:]):
        if hi == lo:
            continue
        edge = [lo, hi - 1, min(lo + 31, hi - 1), min(lo + 32, hi - 1), min(lo + 63, hi - 1), min(lo + 64, hi - 1)]
        for t in set(edge) | set(rng.integers(lo, hi, 60).tolist()):
            for h in {0, Hq - 1, int(rng.integers(Hq))}:
                g = h // (Hq // Hkv)
                ref, ref_lse, A, S = P.prompt_row(q[t, h], k[lo:t + 1, g], v[lo:t + 1, g], D ** -0.5)
                u = (2 * D * S + 2 * (t + 1 - lo) + 16) * U
                assert (np.abs(out[t, h] - ref) <= u * A + 2 * 2.0 ** -8 * A + 2.0 ** -8 * np.abs(ref)).all(), (t, h)
                assert got_lse is None or abs(got_lse[t, h] - ref_lse) <= u + 2 * U * abs(ref_lse), (t, h)


@pytest.mark.parametrize("first", [0, 5])
def test_scores_of_minus_infinity_have_no_weight(lib, first):
    """Keys whose products are -inf (bf16 holds it) count nothing, also where they come first; a row of nothing else is zero."""
    import torch
    for dtype in ("bf16", "f32"):
        q, k, v = _inputs(90, 4, 2, 64, dtype, 17)
        q[..., 0] = 1.0
        k[first:first + 40, :, 0] = float("-inf")
        cu = torch.tensor([0, 90], dtype=torch.int32, device="cuda")
        out, lse = lib.prompt_attention(q, k, v, cu, 0.125, want_lse=True)
        assert torch.isfinite(out).all()
        keep = [t for t in range(90) if not first <= t < first + 40]
        for t in (first + 3, first + 39, 70, 89):
            own = [u for u in keep if u <= t]
            for h in (0, 3):
                if not own:
                    assert (out[t, h] == 0).all() and lse[t, h] == float("-inf")
                    continue
                ref, ref_lse, A, S = P.prompt_row(_f64(q[t, h]), _f64(k[own, h // 2]), _f64(v[own, h // 2]), 0.125)
                u = (2 * 64 * S + 2 * len(own) + 16) * U
                tol = u * A + (2 * 2.0 ** -8 * A + 2.0 ** -8 * np.abs(ref) if dtype == "bf16" else U * np.abs(ref))
                assert (np.abs(_f64(out[t, h]) - ref) <= tol).all()
                assert abs(float(lse[t, h]) - ref_lse) <= u + 2 * U * abs(ref_lse)


def test_many_prompts(lib):
    """More prompts than a wavefront has lanes; empty ones among them."""
    import torch
    lens = np.random.default_rng(1).integers(0, 9, 700)
    lens[[0, 65, 300, 699]] = 0, 150, 70, 0
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    q, k, v = _inputs(int(cu[-1]), 4, 2, 64, "bf16", 5)
    out, lse = lib.prompt_attention(q, k, v, torch.from_numpy(cu).cuda(), 0.125, want_lse=True)
    _check(out, lse, q, k, v, cu, 0.125, "bf16")


def test_sharp_and_growing_scores(lib):
    """Scores that rise along the prompt move the running maximum in every tile; scores of hundreds leave one key."""
    import torch
    cu = np.array([0, 400], np.int32)
    for dtype in ("bf16", "f32"):
        q, k, v = _inputs(400, 4, 2, 64, dtype, 9, k_scale=6.0)
        k *= torch.linspace(0.1, 4, 400).view(-1, 1, 1).cuda().to(k.dtype)
        out, lse = lib.prompt_attention(q, k, v, torch.from_numpy(cu).cuda(), 0.5, want_lse=True)
        _check(out, lse, q, k, v, cu, 0.5, dtype)


def test_equal_values_come_out_as_they_are(lib):
    """Whatever the weights: they are divided by the sum of what entered the product."""
    import torch
    cu = torch.tensor([0, 333], dtype=torch.int32, device="cuda")
    q, k, v = _inputs(333, 4, 2, 128, "bf16", 10)
    v.fill_(1.25)
    out = lib.prompt_attention(q, k, v, cu, 128 ** -0.5)
    assert torch.equal(out, torch.full_like(out, 1.25))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("poison", [float("inf"), float("-inf"), float("nan")])
def test_what_later_tokens_hold_never_enters(lib, dtype, poison):
    import torch
    lens = [90, 50]
    cu = np.array([0, 90, 140], np.int32)
    q, k, v = _inputs(140, 8, 2, 64, dtype, 11)
    out0, lse0 = lib.prompt_attention(q, k, v, torch.from_numpy(cu).cuda(), 0.125, want_lse=True)
    q2, k2, v2 = q.clone(), k.clone(), v.clone()
    for t in (q2, k2, v2):
        t[57] = poison
        t[139] = poison
    out, lse = lib.prompt_attention(q2, k2, v2, torch.from_numpy(cu).cuda(), 0.125, want_lse=True)
    clean = list(range(57)) + list(range(90, 139))
    tol = 2.0 ** -7 if dtype == "bf16" else 1e-5       # (a row evaluated anew sums in another order: the oracle's bound, below)
    assert (out[clean].float() - out0[clean].float()).abs().max() <= tol * out0.float().abs().max()
    # not bit for bit: row 57's infinite maximum makes its wavefront take the exponentials of all its rows against their newest
    # maxima, and each of the two sums of at most 90 weights then rounds on its own ((90 + 8) u each)
    assert (lse[clean] - lse0[clean]).abs().max() <= 2 * (90 + 8) * U + 2 * U * lse0.abs().max()
    part = np.array([0, 57], np.int32)
    _check(out[:57], lse[:57], q[:57], k[:57], v[:57], part, 0.125, dtype)
    assert not torch.isfinite(out[57]).any()           # its own key or value: infinite or NaN
    assert sum(lens) == 140


def test_strided_parts_of_a_projection_and_rows_of_no_prompt(lib):
    import torch
    for dtype, dt in (("bf16", torch.bfloat16), ("f32", torch.float32)):
        fused = torch.randn((77, 8 + 2 + 2, 64), generator=torch.Generator().manual_seed(12)).to(dt).cuda()
        q, k, v = fused[:, :8], fused[:, 8:10], fused[:, 10:]
        cu = np.array([5, 30, 30, 71], np.int32)
        wide = torch.full((77, 9, 64), 7.0, dtype=dt, device="cuda")
        lse = torch.full((77, 8), 7.0, device="cuda")
        out, _ = lib.prompt_attention(q, k, v, torch.from_numpy(cu).cuda(), 0.125, out=wide[:, :8], lse=lse)
        assert out.data_ptr() == wide.data_ptr()
        _check(out, lse, q, k, v, cu, 0.125, dtype)
        for x in (wide[:5], wide[71:], wide[:, 8:], lse[:5], lse[71:]):
            assert (x == 7.0).all()


@pytest.mark.parametrize("cu", [[0, 20, 10, 40], [-3, 20, 40, 40], [0, 20, 41, 41], [0, 20, 2 ** 31 - 1, 40], [40, 0, 0, 0]])
def test_offsets_that_are_no_running_sum_write_nothing(lib, cu):
    import torch
    q, k, v = _inputs(40, 4, 2, 64, "bf16", 13)
    for many in (1, 30):                # the second form of the search, too
        c = torch.tensor(cu[:-1] * many + cu[-1:], dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 3.0)
        lib.prompt_attention(q, k, v, c, 0.125, out=out)
        assert (out == 3.0).all()


def test_no_prompts(lib):
    import torch
    q, k, v = _inputs(4, 4, 2, 64, "bf16", 14)
    out = torch.full_like(q, 3.0)
    lib.prompt_attention(q, k, v, torch.zeros(1, dtype=torch.int32, device="cuda"), 0.125, out=out)
    lib.prompt_attention(q, k, v, torch.zeros(5, dtype=torch.int32, device="cuda"), 0.125, out=out)
    assert (out == 3.0).all()
    assert lib.prompt_attention(q[:0], k[:0], v[:0], torch.zeros(2, dtype=torch.int32, device="cuda"), 0.125).shape == (0, 4, 64)


def test_captured_and_on_another_stream(lib):
    """Replays follow the offsets and values that the buffers hold when they run; two streams at once."""
    import torch
    q, k, v = _inputs(300, 8, 2, 128, "bf16", 15)
    cu = torch.tensor([0, 100, 300], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lib.prompt_attention(q, k, v, cu, 0.1, out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.prompt_attention(q, k, v, cu, 0.1, out=out)
    for i, offsets in enumerate([[0, 100, 300], [0, 299, 300], [17, 17, 250]]):
        cu.copy_(torch.tensor(offsets, dtype=torch.int32))
        q.mul_(-1.0 if i else 1.0)
        want = torch.zeros_like(q)
        lib.prompt_attention(q, k, v, cu, 0.1, out=want)
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            again = lib.prompt_attention(k, k, v, cu, 0.1)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        other = torch.empty_like(again)
        lib.prompt_attention(k, k, v, cu, 0.1, out=other)
        own = slice(offsets[0], offsets[-1])
        assert torch.equal(other[own], again[own])


def test_the_last_row_of_a_large_call_is_reached(lib):
    """Offsets that pass 32 bits: the tokens of a strided view lie far apart."""
    import torch
    T, stride = 66000, 1 << 16
    far = torch.empty((T - 1) * stride + 64, dtype=torch.bfloat16, device="cuda")          # 8.6 GB
    k = far.as_strided((T, 1, 64), (stride, 64, 1))
    g = torch.Generator().manual_seed(16)
    tail = 40
    k[-tail:] = torch.randn((tail, 1, 64), generator=g).bfloat16().cuda()
    q = torch.zeros((T, 1, 64), dtype=torch.bfloat16, device="cuda")
    q[-tail:] = torch.randn((tail, 1, 64), generator=g).bfloat16().cuda()
    cu = torch.tensor([T - tail, T], dtype=torch.int32, device="cuda")
    out, lse = lib.prompt_attention(q, k, k, cu, 0.125, want_lse=True)
    c = lambda x: x[-tail:].contiguous()
    _check(c(out), c(lse), c(q), c(k), c(k), np.array([0, tail], np.int32), 0.125, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_apart(lib, dtype):
    """Offsets between the 64 keys of a stage that need all of 32 bits, and beyond them 64."""
    import torch
    cu, D, stride = np.array([0, 3, 133], np.int32), 64, (1 << 24) - 8
    q, k, v = _inputs(133, 2, 1, D, dtype, 9)
    store = torch.empty(132 * stride + 2 * D, dtype=q.dtype, device="cuda")       # 4.4 or 8.9 GB
    far = [store.as_strided((133, 1, D), (stride, D, 1), o) for o in (0, D)]
    far[0].copy_(k)
    far[1].copy_(v)
    out, lse = lib.prompt_attention(q, *far, torch.from_numpy(cu).cuda(), D ** -0.5, want_lse=True)
    near = lib.prompt_attention(q, k, v, torch.from_numpy(cu).cuda(), D ** -0.5, want_lse=True)
    assert torch.equal(out, near[0]) and torch.equal(lse, near[1])
    with pytest.raises(B.SmartError):
        lib.prompt_attention(q[:2], store.as_strided((2, 1, D), (1 << 24, D, 1)), v[:2], torch.tensor([0, 2], dtype=torch.int32).cuda(), 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_thousands_of_prompts(lib, dtype):
    """Most of them empty or of one token (whose row is its value)."""
    import torch
    lens = np.random.default_rng(5).integers(0, 3, 5000)
    lens[[17, 4000]] = 70, 150
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    q, k, v = _inputs(int(cu[-1]), 4, 2, 64, dtype, 10)
    out, lse = lib.prompt_attention(q, k, v, torch.from_numpy(cu).cuda(), 0.125, want_lse=True)
    _check(out, lse, q, k, v, cu, 0.125, dtype)
