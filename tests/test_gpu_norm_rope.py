"""GPU parity of tree_norm_rope with the binary64 oracle.

Bounds per element (u = 2^-24, M = the sum of |y| over the pair it belongs to): a sum of D squares is off by D u of itself, of
which its root takes half; mean, eps, root and the two products 6 u; cosine and sine 4 u (an angle of at most half a quarter turn in
binary32, two units in their last place); their products and sum 2 u: in all (D / 2 + 12) u M, and the result's own rounding."""
import ctypes

import numpy as np
import pytest

from oracle import norm_rope as N
from oracle import rope as R
from paper_2604_09731_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return B.SmartTree(0)


def _f64(t):
    return t.double().cpu().numpy()


def _type(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _check(got, x, w, pos, eps, base, rot, pairing, dtype):
    ref, mixed = N.norm_rope(_f64(x), None if w is None else _f64(w), pos, eps, base, rot, pairing)
    off = (x.shape[-1] / 2 + 12) * U * mixed
    tol = off + (2.0 ** -8 if dtype == "bf16" else U) * (np.abs(ref) + off)
    err = np.abs(_f64(got) - ref)
    assert (err <= tol).all(), np.nanmax(err / np.maximum(tol, 1e-300))


def _projection(N_, Hq, Hkv, D, dtype, seed, pad=0):
    """Queries and keys inside one projection's output, as a model has them."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((N_, (Hq + 2 * Hkv) * D + pad), generator=g) * 3).to(_type(dtype)).cuda()
    q = x[:, :Hq * D].unflatten(1, (Hq, D))
    k = x[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D))
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(_type(dtype)).cuda() for _ in range(2)]
    return q, k, w


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", [B.SMART_ROPE_HALF_SPLIT, B.SMART_ROPE_INTERLEAVED])
@pytest.mark.parametrize("D,rot", [(128, 128), (64, 64), (128, 64), (96, 48), (80, 80), (80, 40), (64, 2), (34, 22), (6, 4), (2, 2)])
def test_against_the_oracle(lib, dtype, pairing, D, rot):
    import torch
    q, k, w = _projection(37, 5, 2, D, dtype, D + rot)
    pos = np.concatenate([[0, 1, 131071, 2 ** 31 - 1, -7], np.random.default_rng(D).integers(0, 131072, 32)]).astype(np.int32)
    gq, gk = lib.tree_norm_rope(torch.from_numpy(pos).cuda(), q, k, w[0], w[1], eps=1e-5, base=500000.0, rotary_dim=rot, pairing=pairing)
    assert gq.is_contiguous() and gk.is_contiguous()
    far = np.array([p if abs(int(p)) < 1 << 20 else 0 for p in pos])
    near = far == pos                       # (the last digits of the farthest positions' angles are beyond binary64 powers)
    for got, x, weight in ((gq, q, w[0]), (gk, k, w[1])):
        _check(got[torch.from_numpy(near)], x[torch.from_numpy(near)], weight, pos[near], 1e-5, 500000.0, rot, pairing, dtype)
        assert torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,Hq,Hkv", [(1, 32, 8), (1, 1, 0), (3, 0, 5), (700, 28, 4), (2100, 8, 8), (5000, 16, 2)])
def test_rows_and_heads(lib, dtype, n, Hq, Hkv):
    import torch
    q, k, w = _projection(n, Hq, Hkv, 64, dtype, n)
    pos = np.random.default_rng(n).integers(0, 9000, n).astype(np.int32)
    gq, gk = lib.tree_norm_rope(torch.from_numpy(pos).cuda(), q, k, w[0], None)
    pick = sorted({0, n - 1, *np.random.default_rng(1).integers(0, n, 20).tolist()})
    for got, x, weight in ((gq, q, w[0]), (gk, k, None)):
        assert torch.isfinite(got).all()
        _check(got[pick], x[pick], weight, pos[pick], 1e-6, 10000.0, 64, R.HALF_SPLIT, dtype)


@pytest.mark.parametrize("pad", [0, 1, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_are_not_aligned_and_results_in_place(lib, dtype, pad):
    import torch
    q, k, w = _projection(19, 4, 2, 128, dtype, 5, pad)
    pos = torch.arange(100, 119, dtype=torch.int32, device="cuda")
    base = q._base if q._base is not None else q
    before = base.clone()
    want = lib.tree_norm_rope(pos, q.contiguous(), k.contiguous(), *w)
    got = lib.tree_norm_rope(pos, q, k, *w)
    tol = 1e-6 if dtype == "f32" else 2.0 ** -7     # (another variant: sums in another order, at most one step of the type)
    for x, y in zip(got, want):
        assert (x - y).abs().max() <= tol * y.abs().max()
    assert torch.equal(base, before)
    q2, k2 = lib.tree_norm_rope(pos, q, k, *w, q_out=q, k_out=k)
    assert q2.data_ptr() == q.data_ptr() and torch.equal(q, got[0]) and torch.equal(k, got[1])
    assert torch.equal(base[:, 6 * 128:], before[:, 6 * 128:])      # the values beside them, and the padding


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ranges(lib, dtype):
    """Heads of zeros, of values whose squares leave binary32 at either end, with an infinity and with a NaN."""
    import torch
    q, k, _ = _projection(8, 3, 1, 64, dtype, 9)
    q, k = q.contiguous(), k.contiguous()
    q[0] = 0
    q[1] *= 1e30
    q[2, 1] *= 1e36
    q[3] *= 1e-30
    q[4, 0, 5] = float("inf")
    q[5, 2, 7] = float("nan")
    pos = torch.full((8,), 3, dtype=torch.int32, device="cuda")
    out = lib.tree_norm_rope(pos, q, k, None, None, eps=1e-6)[0]
    assert not out[0].any()
    fine = [1, 2, 3, 6, 7]
    _check(out[fine], q[fine], None, [3] * 5, 1e-6, 10000.0, 64, R.HALF_SPLIT, dtype)
    hit = torch.zeros(64, dtype=torch.bool)
    hit[[5, 37]] = True                                             # its pair; the others are x / infinity
    assert out[4, 0].isnan().cpu().tolist() == hit.tolist() and not out[4, 0][~hit].any() and torch.isfinite(out[4, 1:]).all()
    assert out[5, 2].isnan().all() and torch.isfinite(out[5, :2]).all()


def test_captured_on_another_stream(lib):
    import torch
    q, k, w = _projection(500, 32, 8, 128, "bf16", 2)
    pos = torch.arange(500, dtype=torch.int32, device="cuda")
    qo, ko = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)
    graph = torch.cuda.CUDAGraph()
    lib.tree_norm_rope(pos, q, k, *w, q_out=qo, k_out=ko)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lib.tree_norm_rope(pos, q, k, *w, q_out=qo, k_out=ko)
    for shift in (0, 7, 90):
        pos.copy_(torch.arange(shift, 500 + shift, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = lib.tree_norm_rope(pos, q, k, *w)
        assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])


def test_tokens_that_lie_far_apart(lib):
    import torch
    T, stride = 700, 1 << 22
    room = torch.empty((T - 1) * stride + 4096, dtype=torch.bfloat16, device="cuda")
    q, k, w = _projection(T, 4, 2, 128, "bf16", 4)
    far = lambda at, H: room.as_strided((T, H, 128), (stride, 128, 1), at)
    qf, kf = far(0, 4), far(1024, 2)
    qf.copy_(q)
    kf.copy_(k)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    want = lib.tree_norm_rope(pos, q, k, *w)
    got = lib.tree_norm_rope(pos, qf, kf, *w, q_out=qf, k_out=kf)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
