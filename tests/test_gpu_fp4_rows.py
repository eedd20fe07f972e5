"""Attention over a 4-bit cache row by row: each against its own bound, which a long prefix beside a short one does not loosen.

Bounds per element, as in test_gpu_prompt_attention.py (A = the row's softmax average of |v|, S = its largest scale * sum |q| |k|, n its
keys, u = 2^-24): (2 D S + 2 n + 16) u A for scores, exponentials and sums; bf16: a weight is off by up to 2^-8 / (1 + 2^-8) of itself,
in the product and in the sum that divides, together by 2^-8 (A + |result|) <= 2 2^-8 A, and the result is rounded by 2^-8 of itself.
The log-sum-exp is that of the unrounded weights: (2 D S + 2 n + 16) u + 2 u of itself."""
import numpy as np
import pytest

from paper_2604_09731_amd import binding as B
from paper_2604_09731_amd import workloads as W
from tests.test_gpu_fp4_cache import _SHAPES, _case, _dev, _trees

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return B.SmartTree(0)


def attend(lib, w, case, cu, parent, lens, bs):
    """The call on a case of test_gpu_fp4_cache._case, and its softmax scale."""
    args, kc, vc, table, _ = case
    d_cu, d_len = _dev(cu), _dev(lens)
    mask = lib.tree_pack(d_cu, _dev(parent), d_len)[3]
    scale = w.head_dim ** -0.5
    return lambda **kw: lib.tree_verify_attention(*args, kc, vc, table, d_len, d_cu, mask, scale, B.SMART_KV_INTERLEAVED, block_size=bs,
                                                  kv_cache_dtype=B.SMART_FP4_E2M1, **kw), scale


def rows(oracle, ref_args, scale):
    """Result, log-sum-exp, A, S and the number of keys of every row."""
    q, kt, vt, kc, vc, table, lens, cu, parent = ref_args
    ref, ref_lse = oracle.tree_attention(*ref_args, scale)
    A, _ = oracle.tree_attention(q, kt, np.abs(vt), kc, np.abs(vc), table, lens, cu, parent, scale)
    S, n = np.zeros(ref.shape[:2]), np.zeros(ref.shape[:2])
    G, bs = q.shape[1] // kt.shape[1], kc.shape[2]
    for b, L in enumerate(lens):
        t = np.arange(int(L))
        keys = np.concatenate([kc[table[b, t // bs], :, t % bs], kt[cu[b]:cu[b + 1]]])          # (all nodes: no less)
        for h in range(q.shape[1]):
            if cu[b + 1] > cu[b]:
                S[cu[b]:cu[b + 1], h] = scale * (np.abs(q[cu[b]:cu[b + 1], h]) @ np.abs(keys[:, h // G]).T).max(1)
        n[cu[b]:cu[b + 1]] = len(keys)
    return ref, ref_lse, A, S, n


def check_rows(out, lse, want, dtype):
    ref, ref_lse, A, S, n = want
    got = out.double().cpu().numpy()
    u = (2 * got.shape[2] * S + 2 * n + 16) * U
    tol = u[..., None] * A + (2 * 2.0 ** -8 * A + 2.0 ** -8 * np.abs(ref) if dtype == "bf16" else U * np.abs(ref))
    assert (np.abs(got - ref) <= tol).all(), np.nanmax(np.abs(got - ref) / tol)
    if lse is not None:
        err = np.abs(lse.double().cpu().numpy() - ref_lse)
        assert (err <= u + 2 * U * np.abs(ref_lse)).all(), np.nanmax(err / u)


@pytest.mark.parametrize("dtype,D,bs,heads,sizes,lens", _SHAPES + [
    ("bf16", 128, 16, (8, 2), [18, 3, 25, 32, 60, 128, 1], [900, 1030, 1337, 129, 641, 1500, 700]),
    ("bf16", 64, 16, (8, 1), [1, 9, 2], [5000, 1, 2000])])
def test_every_row(lib, oracle_attention, dtype, D, bs, heads, sizes, lens):
    import torch
    w = W.Workload("fp4", dtype, len(sizes), heads[0], heads[1], D, 0, 0, seed=31)
    cu, parent = _trees(sizes)
    lens = np.array(lens, np.int32)
    case = _case(w, cu, parent, lens, bs, 60, spare_bytes=16)
    call, scale = attend(lib, w, case, cu, parent, lens, bs)
    want = rows(oracle_attention, case[4], scale)
    for workers in (0, 1, 7):
        lib.set_option(B.SMART_OPT_TVA_WORKERS, workers)
        try:
            out, lse = call(want_lse=True)
            bare = call()
        finally:
            lib.set_option(B.SMART_OPT_TVA_WORKERS, 0)
        check_rows(out, lse, want, dtype)
        check_rows(bare, None, want, dtype)
    out, lse = call(static=True, h_cu_nodes=cu, out=torch.empty_like(out), lse=torch.empty_like(lse))
    check_rows(out, lse, want, dtype)
    bare = call(static=True, h_cu_nodes=cu, out=torch.empty_like(out))
    check_rows(bare, None, want, dtype)


@pytest.mark.parametrize("D,nodes", [(128, 1), (128, 12), (128, 30), (64, 1), (64, 30)])
@pytest.mark.parametrize("lse", [False, True])
def test_equal_values_come_out_as_they_are(lib, D, nodes, lse):
    """Whatever the weights: they are divided by the sum of what entered the product.  Token 300 has 128.49 times the weight of token
    32, against which it is taken, and 128.49 is off by half a step in bf16; no other key counts (2^-112)."""
    import torch
    Hq, Hkv, bs, n = 8, 2, 16, 600
    k = torch.zeros((n, Hkv, D), dtype=torch.bfloat16, device="cuda")
    k[..., 0] = -16.0
    k[32, :, 0], k[300, :, 0] = 0.0, 1.0
    v = torch.full_like(k, 1.5)
    blocks = (n + bs - 1) // bs
    kc, vc = (torch.zeros((blocks, Hkv, B.fp4_page_bytes(bs, D)), dtype=torch.uint8, device="cuda") for _ in range(2))
    lib.kv_cache_write_fp4(k, v, _dev(np.arange(n).astype(np.int64)), kc, vc, bs)
    q = torch.zeros((nodes, Hq, D), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    cu, parent = _trees([nodes])
    length = _dev(np.array([n], np.int32))
    mask = lib.tree_pack(_dev(cu), _dev(parent), length)[3]
    scale = float(np.log(128.49))
    for static in (False, True):
        got = lib.tree_verify_attention(q, k[:nodes].contiguous(), v[:nodes].contiguous(), kc, vc, _dev(np.arange(blocks).reshape(1, -1), np.int32),
                                        length, _dev(cu), mask, scale, B.SMART_KV_INTERLEAVED, block_size=bs, want_lse=lse,
                                        static=static, kv_cache_dtype=B.SMART_FP4_E2M1)
        out = got[0] if lse else got
        assert torch.equal(out, torch.full_like(out, 1.5)), (out.min().item(), out.max().item())
        if lse:
            assert (got[1].double() - np.log(129.49)).abs().max() <= 1e-5
