"""GPU parity of prompt_attention with a window with the binary64 oracle; bounds as in test_gpu_prompt_attention.py, with a row's
own number of keys."""
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


def _cu(lens, first=0):
    import torch
    cu = (first + np.concatenate([[0], np.cumsum(lens)])).astype(np.int32)
    return cu, torch.from_numpy(cu).cuda()


def _check_rows(out, lse, q, k, v, cu, window, sinks, dtype, rows):
    """rows: (prompt, token in it, head)."""
    D, G = q.shape[2], q.shape[1] // k.shape[1]
    scale = D ** -0.5
    for b, t, h in rows:
        lo, own = cu[b], cu[b] + np.array(P.seen(t, window, sinks))
        ref, ref_lse, A, S = P.prompt_row(q[lo + t, h], k[own, h // G], v[own, h // G], scale)
        u = (2 * D * S + 2 * len(own) + 16) * U
        tol = u * A + (2 * 2.0 ** -8 * A + 2.0 ** -8 * np.abs(ref) if dtype == "bf16" else U * np.abs(ref))
        err = np.abs(out[lo + t, h] - ref)
        assert (err <= tol).all(), (b, t, h, np.max(err / tol))
        assert lse is None or abs(lse[lo + t, h] - ref_lse) <= u + 2 * U * abs(ref_lse), (b, t, h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 8, 2), (128, 4, 4), (128, 7, 1)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (2, 1), (31, 0), (32, 4), (64, 64), (65, 7), (100, 130), (5, 40), (1000, 2), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_against_the_oracle(lib, dtype, D, Hq, Hkv, window, sinks):
    lens = [129, 0, 1, 300, 40]
    cu, d_cu = _cu(lens)
    q, k, v = _inputs(int(cu[-1]), Hq, Hkv, D, dtype, window % 1000 + sinks % 1000)
    out, lse = lib.prompt_attention(q, k, v, d_cu, D ** -0.5, want_lse=True, window=window, sinks=sinks)
    bare = lib.prompt_attention(q, k, v, d_cu, D ** -0.5, window=window, sinks=sinks)
    import torch
    assert torch.equal(bare, out)
    rows = [(b, t, h) for b, n in enumerate(lens) for t in range(n) for h in sorted({0, Hq - 1, t % Hq})]
    _check_rows(_f64(out), _f64(lse), _f64(q), _f64(k), _f64(v), cu, window, sinks, dtype, rows)


@pytest.mark.parametrize("dtype,D,Hq,Hkv,lens,window,sinks", [
    ("bf16", 128, 28, 4, [1500, 2, 700], 333, 5), ("bf16", 64, 32, 8, [1500, 2, 700], 500, 0), ("bf16", 128, 64, 8, [3000, 1, 0, 1200, 77], 1024, 4),
    ("bf16", 64, 64, 8, [3000, 1, 0, 1200, 77], 64, 100), ("bf16", 128, 16, 16, [2500], 200, 1), ("bf16", 64, 16, 16, [2500], 7, 64),
    ("bf16", 128, 64, 8, [5000], 40, 4), ("f32", 64, 8, 2, [2000, 300], 257, 3), ("f32", 128, 8, 8, [1100], 96, 65),
    ("bf16", 128, 8, 2, [70] * 90, 33, 2), ("bf16", 128, 32, 8, [37], 8, 4)])
@pytest.mark.parametrize("want_lse", [False, True])
def test_large_calls_by_some_of_their_rows(lib, dtype, D, Hq, Hkv, lens, window, sinks, want_lse):
    cu, d_cu = _cu(lens)
    q, k, v = _inputs(int(cu[-1]), Hq, Hkv, D, dtype, 31)
    got = lib.prompt_attention(q, k, v, d_cu, D ** -0.5, want_lse=want_lse, window=window, sinks=sinks)
    out, lse = (_f64(got[0]), _f64(got[1])) if want_lse else (_f64(got), None)
    assert np.isfinite(out).all()
    rng = np.random.default_rng(0)
    rows = []
    for b, n in enumerate(lens):
        edge = {0, n - 1, window - 1, window, window + 1, window + sinks, window + sinks - 1, window + sinks + 63, window + 64, sinks, sinks + 1}
        picks = {t for t in edge if 0 <= t < n} | set(rng.integers(0, n, 40 if n > 200 else 3).tolist() if n else [])
        rows += [(b, t, h) for t in sorted(picks) for h in {0, Hq - 1, int(rng.integers(Hq))}]
    _check_rows(out, lse, _f64(q), _f64(k), _f64(v), cu, window, sinks, dtype, rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_what_a_window_has_left_never_enters(lib, dtype, D, bad):
    """Rows whose window has left a token do not see what it holds; rows that see it are what the whole formula gives."""
    import torch
    T, window, sinks, at = 400, 50, 6, 130
    cu, d_cu = _cu([T])
    q, k, v = _inputs(T, 8, 2, D, dtype, 5)
    clean = lib.prompt_attention(q, k, v, d_cu, D ** -0.5, want_lse=True, window=window, sinks=sinks)
    v2, k2 = v.clone(), k.clone()
    v2[at] = bad
    k2[at] = bad
    for kx, vx in ((k, v2), (k2, v)):
        out, lse = lib.prompt_attention(q, kx, vx, d_cu, D ** -0.5, want_lse=True, window=window, sinks=sinks)
        blind = [t for t in range(T) if at not in P.seen(t, window, sinks)]
        tol = U * 2000 if dtype == "f32" else 2.0 ** -7
        assert (out[blind].float() - clean[0][blind].float()).abs().max() <= tol * clean[0].float().abs().max()
        assert (lse[blind] - clean[1][blind]).abs().max() <= 1e-4
        if vx is v2:
            seeing = [t for t in range(T) if t not in blind]
            assert not torch.isfinite(out[seeing]).any() and torch.isfinite(lse).all()


def test_masked_scores_inside_a_window(lib):
    """Keys whose scores are -infinity count nothing; a row whose window holds nothing else is zero."""
    import torch
    for dtype in ("bf16", "f32"):
        q, k, v = _inputs(200, 4, 2, 64, dtype, 17)
        q[..., 0] = 1.0
        k[60:140, :, 0] = float("-inf")
        _, d_cu = _cu([200])
        out, lse = lib.prompt_attention(q, k, v, d_cu, 0.125, want_lse=True, window=20, sinks=0)
        assert torch.isfinite(out).all()
        assert not out[79:140].any() and (lse[79:140] == float("-inf")).all() and torch.isfinite(lse[:79]).all()
        part = lib.prompt_attention(q, k, v, d_cu, 0.125, window=20, sinks=2)
        assert part[79:140].any(-1).all()


def test_parts_of_a_projection_rows_of_no_prompt_and_a_graph(lib):
    import torch
    T, Hq, Hkv, D = 700, 8, 2, 128
    x = torch.randn((T, (Hq + 2 * Hkv) * D), generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    q, k, v = (p.unflatten(1, (-1, D)) for p in x.split([Hq * D, Hkv * D, Hkv * D], 1))
    cu, d_cu = _cu([300, 350], 20)
    out = torch.full((T, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lib.prompt_attention(q, k, v, d_cu, D ** -0.5, out=out, window=100, sinks=4)
    assert (out[:20] == 7).all() and (out[670:] == 7).all()
    want = lib.prompt_attention(q.contiguous(), k.contiguous(), v.contiguous(), d_cu, D ** -0.5, window=100, sinks=4)
    assert torch.equal(out[20:670], want[20:670])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.prompt_attention(q, k, v, d_cu, D ** -0.5, out=out, window=100, sinks=4)
    for _ in range(3):
        x.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[20:670], lib.prompt_attention(q, k, v, d_cu, D ** -0.5, window=100, sinks=4)[20:670])


def test_bad_offsets_write_nothing(lib):
    import torch
    q, k, v = _inputs(50, 4, 2, 64, "bf16", 1)
    for offsets in ([0, 60], [-1, 50], [30, 20]):
        out = torch.full_like(q, 3.0)
        lib.prompt_attention(q, k, v, torch.tensor(offsets, dtype=torch.int32, device="cuda"), 0.125, out=out, window=5, sinks=1)
        assert (out == 3).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_that_lie_far_apart(lib, dtype):
    """Offsets past 32 bits: where the first tokens and the window are more than that apart, the gap begins with a stage."""
    import torch
    dt, T, stride = (torch.bfloat16 if dtype == "bf16" else torch.float32), 1100, 1 << 22
    room = torch.empty((T - 1) * stride + 4096, dtype=dt, device="cuda")
    far = lambda at, H: room.as_strided((T, H, 64), (stride, 64, 1), at)
    q, k, v = _inputs(T, 8, 2, 64, dtype, 41)
    qf, kf, vf = far(0, 8), far(1024, 2), far(2048, 2)
    for x, y in ((qf, q), (kf, k), (vf, v)):
        x.copy_(y)
    _, d_cu = _cu([T])
    cu = np.array([0, T])
    for window, sinks in ((100, 5), (64, 64), (300, 130)):
        out, lse = lib.prompt_attention(qf, kf, vf, d_cu, 0.125, want_lse=True, window=window, sinks=sinks)
        rows = [(0, t, h) for t in (0, 5, window, window + sinks, window + sinks + 64, 700, 1023, 1024, T - 1) for h in (0, 7)]
        _check_rows(_f64(out), _f64(lse), _f64(q), _f64(k), _f64(v), cu, window, sinks, dtype, rows)
