"""Attention over a 4-bit cache where rows are evaluated a second time, key by key: products past binary32, infinities and NaN that a row
does not see, cached values that are NaN, offsets that do not ascend.  Bounds as in test_gpu_fp4_rows.py."""
import functools

import numpy as np
import pytest

from paper_2604_09731_amd import binding as B
from paper_2604_09731_amd import workloads as W
from oracle import fp4 as F
from tests.test_gpu_fp4_cache import _case, _dev, _trees
from tests.test_gpu_fp4_rows import attend, check_rows, rows

pytestmark = pytest.mark.gpu
FORMS = [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)]
BIG = 6 * 2.0 ** 125                                # the largest value that is stored


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return B.SmartTree(0)


@pytest.mark.parametrize("dtype,D", FORMS)
@pytest.mark.parametrize("nodes", [1, 12, 30])
@pytest.mark.parametrize("static", [False, True])
def test_the_largest_stored_value_under_a_weight_above_one(lib, dtype, D, nodes, static):
    """Token 300 holds it and has 2^7.5 times the weight of token 32, against which it is taken where one wavefront comes to both:
    their product is past binary32, the row is not.  No other key counts (2^-120)."""
    import torch
    Hq, Hkv, bs, n = 8, 2, 16, 600
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    k = torch.zeros((n, Hkv, D), dtype=dt, device="cuda")
    k[..., 0] = -16.0
    k[32, :, 0], k[300, :, 0] = 0.0, 1.0
    v = torch.ones_like(k)
    v[300] = BIG
    v[300, 1] = -BIG
    blocks = (n + bs - 1) // bs
    kc, vc = (torch.zeros((blocks, Hkv, B.fp4_page_bytes(bs, D)), dtype=torch.uint8, device="cuda") for _ in range(2))
    lib.kv_cache_write_fp4(k, v, _dev(np.arange(n).astype(np.int64)), kc, vc, bs)
    assert lib.kv_cache_read_fp4(_dev(np.array([300], np.int64)), kc, vc, D, bs, dt)[1][0, 0, 5].item() == BIG
    q = torch.zeros((nodes, Hq, D), dtype=dt, device="cuda")
    q[..., 0] = 1.0
    cu, parent = _trees([nodes])
    length = _dev(np.array([n], np.int32))
    mask = lib.tree_pack(_dev(cu), _dev(parent), length)[3]
    lib.set_option(B.SMART_OPT_TVA_WORKERS, 1)      # (the split form: all of a segment in one piece)
    try:
        out, lse = lib.tree_verify_attention(q, k[:nodes].contiguous(), torch.ones_like(k[:nodes]), kc, vc,
                                             _dev(np.arange(blocks).reshape(1, -1), np.int32), length, _dev(cu), mask,
                                             float(7.5 * np.log(2.0)), B.SMART_KV_INTERLEAVED, block_size=bs, want_lse=True, static=static,
                                             kv_cache_dtype=B.SMART_FP4_E2M1)
    finally:
        lib.set_option(B.SMART_OPT_TVA_WORKERS, 0)
    want = BIG * (2.0 ** 7.5 / (1 + 2.0 ** 7.5))
    got = out.double().cpu().numpy()
    tol = 2.0 ** -8 * want + 2 * 2.0 ** -8 * want if dtype == "bf16" else 1e-5 * want
    assert (np.abs(got[:, :4] - want) <= tol).all() and (np.abs(got[:, 4:] + want) <= tol).all()
    assert (lse.double() - np.log(1 + 2.0 ** 7.5)).abs().max() <= 1e-5


def _ancestors(cu, parent, b):
    """sees[i, j]: node i of tree b sees node j."""
    n = cu[b + 1] - cu[b]
    sees = np.zeros((n, n), bool)
    for i in range(n):
        j = i
        while j >= 0:
            sees[i, j] = True
            j = parent[cu[b] + j]
    return sees


@functools.lru_cache(maxsize=None)
def _shared_case(oracle, dtype, D, sizes, lens):
    """Inputs that no test changes, and their rows' results and bounds."""
    w = W.Workload("fp4", dtype, len(sizes), 8, 2, D, 0, 0, seed=31)
    cu, parent = _trees(list(sizes))
    lens = np.array(lens, np.int32)
    case = _case(w, cu, parent, lens, 16, 61)
    return w, cu, parent, lens, case, rows(oracle, case[4], D ** -0.5)


@pytest.mark.parametrize("dtype,D", FORMS)
@pytest.mark.parametrize("sizes,lens", [((1, 3, 9), (40, 300, 0)), ((17, 40), (700, 130)), ((128, 33, 2), (520, 1, 90))])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_what_one_node_holds_reaches_only_its_descendants(lib, oracle_attention, dtype, D, sizes, lens, bad):
    """A value of one node, then a key: rows that do not see it stay within their bounds, rows that do are infinite or NaN in that head
    dim (value) or NaN (key)."""
    import torch
    w, cu, parent, lens, case, (ref, ref_lse, A, S, n) = _shared_case(oracle_attention, dtype, D, sizes, lens)
    q, kt, vt = case[0]
    for b, node in ((0, sizes[0] // 3), (0, sizes[0] - 1), (1, sizes[1] // 2)):
        sees = np.zeros(len(ref), bool)
        sees[cu[b]:cu[b + 1]] = _ancestors(cu, parent, b)[:, node]
        at = cu[b] + node
        for which in ("value", "key"):
            kt2, vt2 = kt.clone(), vt.clone()
            if which == "value":
                vt2[at, :, 5], vt2[at, :, D - 2] = bad, -bad
            else:
                kt2[at, :, 9] = bad if np.isnan(bad) else float("nan")
            call, _ = attend(lib, w, ((q, kt2, vt2),) + case[1:], cu, parent, lens, 16)
            for kw in (dict(), dict(static=True, h_cu_nodes=cu)):
                out, lse = call(want_lse=True, **kw)
                check_rows(out[~sees], lse[~sees], tuple(x[~sees] for x in (ref, ref_lse, A, S, n)), dtype)
                got = out[sees].double().cpu().numpy()
                if which == "key":
                    assert np.isnan(got).all()
                    continue
                assert not np.isfinite(got[..., [5, D - 2]]).any()
                if not np.isnan(bad):                   # (all weights here are far from underflowing)
                    assert (got[..., 5] == bad).all() and (got[..., D - 2] == -bad).all()
                keep = [d for d in range(D) if d not in (5, D - 2)]
                check_rows(torch.from_numpy(got[..., keep]), lse[sees],
                           (ref[sees][..., keep], ref_lse[sees], A[sees][..., keep], S[sees], n[sees]), dtype)


@pytest.mark.parametrize("dtype,D", FORMS)
def test_cached_values_that_are_NaN_stay_in_their_32_head_dims(lib, oracle_attention, dtype, D):
    w = W.Workload("fp4", dtype, 3, 8, 2, D, 0, 0, seed=31)
    cu, parent = _trees([3, 40, 5])
    lens = np.array([700, 1100, 90], np.int32)
    case = _case(w, cu, parent, lens, 16, 62)
    call, scale = attend(lib, w, case, cu, parent, lens, 16)
    want = rows(oracle_attention, case[4], scale)
    table = case[3].cpu().numpy()
    for token in (0, 333, 1099):                        # kv head 1 of sequence 1
        case[2][int(table[1, token // 16]), 1, F.scale_at("v", token % 16, 33, 16, D)] = 255
    hit = np.zeros(want[0].shape, bool)
    hit[cu[1]:cu[2], 4:, 32:64] = True
    for kw in (dict(), dict(static=True, h_cu_nodes=cu)):
        out, lse = call(want_lse=True, **kw)
        got = out.double().cpu().numpy()
        assert np.isnan(got[hit]).all() and np.isfinite(got[~hit]).all()
        out = out.double().cpu()
        out[hit] = 0.0
        check_rows(out, lse, (np.where(hit, 0.0, want[0]),) + want[1:], dtype)


@pytest.mark.parametrize("dtype,D", FORMS)
@pytest.mark.parametrize("static", [False, True])
def test_offsets_that_are_not_ascending(lib, dtype, D, static):
    """Every row has the one owner that the general kernel finds, and its value; both hold weights in binary32 then, and a bf16 result
    is rounded by each (2^-8 of itself)."""
    import torch
    for sizes, lens, offsets in (([5, 20, 70, 3, 9], [100, 333, 64, 0, 50], [0, 25, 5, 95, 98, 107]), ([30, 40], [70, 90], [40, 0, 70]),
                                 ([2] * 65, [7 * i % 90 for i in range(65)], list(range(130, -1, -2)))):
        cu, parent = _trees(sizes)
        lens = np.array(lens, np.int32)
        g = torch.Generator().manual_seed(63)
        blocks, N = [(int(m) + 15) // 16 for m in lens], int(cu[-1])
        kc, vc = (torch.randint(0, 256, (sum(blocks) + 1, 2, B.fp4_page_bytes(16, D)), generator=g).to(torch.uint8) for _ in range(2))
        for c in (kc, vc):
            c[..., 8 * D:] = 125                          # (scales of 1 / 4: values up to 1.5)
        kc, vc = kc.cuda(), vc.cuda()
        table = np.full((len(lens), max(blocks)), -9, np.int32)
        for b, first in enumerate(np.cumsum(blocks) - blocks):
            table[b, :blocks[b]] = np.arange(first, first + blocks[b])
        table = _dev(table)
        args = [torch.randn((N, h, D), generator=g).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda() for h in (8, 2, 2)]
        mask = lib.tree_pack(_dev(cu), _dev(parent), _dev(lens))[3]
        d_cu = _dev(np.array(offsets, np.int32))
        got = []
        for general in (1, 0):
            lib.set_option(B.SMART_OPT_TVA_FORCE_GENERAL, general)
            try:
                got.append(lib.tree_verify_attention(*args, kc, vc, table, _dev(lens), d_cu, mask, D ** -0.5, B.SMART_KV_INTERLEAVED,
                                                     out=torch.full_like(args[0], 7.0), want_lse=True, static=static and not general,
                                                     kv_cache_dtype=B.SMART_FP4_E2M1))
            finally:
                lib.set_option(B.SMART_OPT_TVA_FORCE_GENERAL, 0)
        (ref, ref_lse), (out, lse) = got
        tol = (2 * 2.0 ** -8 if dtype == "bf16" else 0.0) * ref.double().abs() + 1e-5 * 5.0     # (|v| of a few: sums of some hundred keys)
        assert ((out.double() - ref.double()).abs() <= tol).all()
        same = ref_lse == lse                             # (-infinity: rows of no sequence)
        assert ((lse - ref_lse).abs()[~same] <= 1e-4).all()
