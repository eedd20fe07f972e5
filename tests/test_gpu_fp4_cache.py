"""GPU parity of the 4-bit KV cache with the CPU oracle: writing, reading and committing are bit-exact; attention is compared
with the binary64 oracle over the decoded cache, so the comparison measures the kernels and not the quantisation."""
import numpy as np
import pytest

from oracle import fp4 as F
from paper_2604_09731_amd import binding as B
from paper_2604_09731_amd import workloads as W
from tests import helpers as H

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return B.SmartTree(0)


def _dev(a, dtype=None):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).to("cuda")


def _rows(n, Hkv, D, dtype, seed):
    """Rows with the values that encoding can go wrong at; what they are in binary64."""
    import torch
    g = np.random.default_rng(seed)
    x = (g.standard_normal((n, Hkv, D)) * np.exp2(g.integers(-6, 7, (n, Hkv, 1)))).astype(np.float32)
    x[0, 0, :10] = [0.0, -0.0, 6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]
    x[0, 0, 10:32] = 0.0
    x[1 % n, 0, :32] = 0.0
    x[2 % n, 0, 5] = np.inf
    x[3 % n, 0, 6] = np.nan
    x[4 % n, 0, 32:64] *= np.float32(2.0 ** -130)
    x[5 % n, 0, 32:64] = np.float32(3e38)
    x[6 % n, 0, 7] = 7.0 * np.abs(x[6 % n, 0, :32]).max()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    t = torch.from_numpy(x).to(dt).cuda()
    return t, t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv,D,bs,nb,n", [(3, 128, 16, 7, 60), (1, 64, 8, 9, 1), (2, 64, 24, 4, 96), (2, 128, 64, 2, 100), (1, 32, 8, 3, 20)])
def test_write_and_read(lib, dtype, Hkv, D, bs, nb, n):
    import torch
    rng = np.random.default_rng(4)
    k, k64 = _rows(n, Hkv, D, dtype, 1)
    v, v64 = _rows(n, Hkv, D, dtype, 2)
    slots = rng.permutation(nb * bs)[:n].astype(np.int64)
    if n > 30:
        slots[8:24] = np.arange(16) + 8                          # whole groups of consecutive slots
        slots[24:] = np.setdiff1d(np.arange(nb * bs), slots[:24])[:n - 24]
        slots[:8] = np.setdiff1d(np.arange(nb * bs), slots[8:])[:8]
        slots[27], slots[28] = -1, nb * bs
    assert len(set(slots.tolist())) == n
    page = B.fp4_page_bytes(bs, D)
    assert page == F.page_bytes(bs, D)
    store = torch.full((nb, Hkv + 1, (page + 31) // 16 * 16), 0x5A, dtype=torch.uint8, device="cuda")       # pages that are parts of larger rows
    kc, vc = store.clone()[:, :Hkv, :page], store.clone()[:, :Hkv, :page]
    want = {}
    for which, x in (("k", k64), ("v", v64)):
        codes, scales = F.encode(x)
        pages = np.full((nb, Hkv, page), 0x5A, np.uint8)
        for t in range(n):
            if 0 <= slots[t] < nb * bs:
                for g in range(Hkv):
                    F.put_row(pages[slots[t] // bs, g], which, slots[t] % bs, codes[t, g], scales[t, g], bs)
        want[which] = pages, F.decode(codes, scales)
    lib.kv_cache_write_fp4(k, v, _dev(slots), kc, vc, bs)
    torch.cuda.synchronize()
    assert np.array_equal(kc.cpu().numpy(), want["k"][0])
    assert np.array_equal(vc.cpu().numpy(), want["v"][0])
    for c in (kc, vc):                                            # nothing beside the pages is touched
        whole = c.as_strided(store.shape, store.stride())
        assert (whole[:, Hkv:] == 0x5A).all() and (whole[:, :, page:] == 0x5A).all()
    for dt in (torch.bfloat16, torch.float32):
        for t, got in zip("kv", lib.kv_cache_read_fp4(_dev(slots), kc, vc, D, bs, dt)):
            ref = np.where(((slots >= 0) & (slots < nb * bs))[:, None, None], want[t][1], 0.0)
            assert np.array_equal(got.double().cpu().numpy(), ref, equal_nan=True)


def test_reading_knows_every_code_and_scale(lib):
    import torch
    bs, D = 16, 128
    rng = np.random.default_rng(6)
    pages = rng.integers(0, 256, (40, 2, F.page_bytes(bs, D))).astype(np.uint8)
    kc, vc = _dev(pages), _dev(pages[::-1].copy())
    slots = np.arange(40 * bs).astype(np.int64)
    got = lib.kv_cache_read_fp4(_dev(slots), kc, vc, D, bs, torch.float32)
    for which, x, p in zip("kv", got, (pages, pages[::-1])):
        ref = F.decode_pages(p, which, bs, D).transpose(0, 2, 1, 3).reshape(-1, 2, D)
        ref = np.where(np.abs(ref) > 3.4e38, np.copysign(np.inf, ref), ref)                   # 4 2^126 and beyond
        assert np.array_equal(x.double().cpu().numpy(), ref, equal_nan=True)


def _case(w, cu, parent, lens, bs, seed, spare_bytes=0):
    """A random 4-bit cache with its decoded values; slots past a prefix hold NaN scales and any codes."""
    import torch
    g = np.random.default_rng(seed)
    B_, D, Hkv = len(lens), w.head_dim, w.num_kv_heads
    blocks = (lens + bs - 1) // bs
    nb = int(blocks.sum()) + 2
    perm = g.permutation(nb).astype(np.int32)
    table = np.full((B_, max(1, int(blocks.max())) + 1), -9, np.int32)
    at = 0
    for b, m in enumerate(blocks):
        table[b, :m] = perm[at:at + m]
        at += int(m)
    pages, values = {}, {}
    for which in "kv":
        x = (g.standard_normal((nb, Hkv, bs, D))).astype(np.float32)
        x[..., 3::41] *= 4.0
        codes, scales = F.encode(x)
        out = np.zeros((nb, Hkv, F.page_bytes(bs, D) + spare_bytes), np.uint8)
        slot, d = np.meshgrid(np.arange(bs), np.arange(D), indexing="ij")
        for low in (0, 1):
            sel = d % 2 == low
            out[:, :, F.code_byte(which, slot, d, bs, D)[sel]] |= codes[..., sel] << (4 * low)
        out[:, :, F.scale_at(which, slot, d, bs, D)] = np.repeat(scales, 32, -1)
        values[which] = F.decode(codes, scales)
        for b in range(B_):                                        # what lies past the prefix in its last block
            for s in range(int(lens[b]) % bs, bs) if lens[b] % bs else ():
                for dd in range(D):
                    out[table[b, blocks[b] - 1], :, F.scale_at(which, s, dd, bs, D)] = 255
        pages[which] = _dev(out)
    N = int(cu[-1])
    dt = w.dtype
    q, kt, vt = (W._normal(seed, i, (N, h, D), 1.0, dt) for i, h in ((1, w.num_q_heads), (2, Hkv), (3, Hkv)))
    f64 = (lambda x: W.bf16_bits_to_f32(x).astype(np.float64)) if dt == "bf16" else (lambda x: x.astype(np.float64))
    args = tuple(H.torch_elems(x, dt, "cuda") for x in (q, kt, vt))
    ref_args = (f64(q), f64(kt), f64(vt), values["k"], values["v"], np.clip(table, 0, nb - 1), lens, cu, parent)
    return args, pages["k"], pages["v"], _dev(table), ref_args


def _trees(sizes, seed=8):
    rng = np.random.default_rng(seed)
    shapes = ["random", "chain", "star"]
    cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    return cu, np.concatenate([W.random_tree(n, rng, shapes[i % 3]) for i, n in enumerate(sizes)]).astype(np.int32)


def _attend(lib, w, case, cu, parent, lens, bs, **kw):
    args, kc, vc, table, ref_args = case
    d_cu, d_len = _dev(cu), _dev(lens)
    mask = lib.tree_pack(d_cu, _dev(parent), d_len)[3]
    scale = w.head_dim ** -0.5
    call = lambda **more: lib.tree_verify_attention(*args, kc, vc, table, d_len, d_cu, mask, scale, B.SMART_KV_INTERLEAVED, block_size=bs,
                                                    kv_cache_dtype=B.SMART_FP4_E2M1, want_lse=True, **dict(kw, **more))
    return call, scale, ref_args


def _check(out, lse, ref, ref_lse, dtype):
    got = H.out_to_f64(out, dtype)
    assert np.isfinite(got).all()
    assert H.rel_err(got, ref) <= (2.0 ** -7 if dtype == "bf16" else H.TOL["f32"]), H.rel_err(got, ref)
    assert np.abs(lse.double().cpu().numpy() - ref_lse).max() <= 1e-4


_SHAPES = [
    # dtype, D, block size, heads, tree sizes, prefixes
    ("bf16", 128, 16, (8, 2), [1, 3, 8, 17, 40, 2, 128], [0, 1, 31, 32, 33, 517, 300]),
    ("bf16", 128, 16, (32, 8), [7], [517]),
    ("bf16", 128, 16, (8, 1), [1, 1, 1, 1], [2000, 1, 64, 1025]),
    ("bf16", 128, 16, (7, 1), [4, 5, 9, 10], [640, 95, 1500, 16]),
    ("bf16", 128, 16, (8, 1), [1, 1, 2], [5000, 1, 4097]),
    ("bf16", 128, 64, (8, 2), [1, 9, 16, 20], [100, 63, 64, 700]),
    ("bf16", 128, 24, (4, 4), [1, 8, 33, 2], [100, 23, 24, 700]),
    ("bf16", 128, 8, (8, 2), [1, 8, 33, 2], [100, 7, 8, 700]),
    ("bf16", 64, 16, (8, 2), [1, 8, 33, 64], [100, 0, 129, 700]),
    ("f32", 128, 16, (8, 2), [1, 8, 33, 64], [100, 0, 129, 700]),
    ("f32", 64, 32, (8, 2), [15, 15, 1, 70], [128, 1, 300, 555]),
    ("f32", 64, 8, (4, 4), [15, 2, 1], [9, 40, 300]),
]


@pytest.mark.parametrize("dtype,D,bs,heads,sizes,lens", _SHAPES)
def test_attention(lib, oracle_attention, dtype, D, bs, heads, sizes, lens):
    import torch
    w = W.Workload("fp4", dtype, len(sizes), heads[0], heads[1], D, 0, 0, seed=31)
    cu, parent = _trees(sizes)
    lens = np.array(lens, np.int32)
    call, scale, ref_args = _attend(lib, w, _case(w, cu, parent, lens, bs, 40, spare_bytes=16), cu, parent, lens, bs)
    ref, ref_lse = oracle_attention.tree_attention(*ref_args, scale)
    status = torch.full((len(sizes),), 7, dtype=torch.int32, device="cuda")
    out, lse = call(status=status)
    _check(out, lse, ref, ref_lse, dtype)
    assert not status.any()
    # the form without a workspace
    out, lse = call(static=True, h_cu_nodes=cu, out=torch.empty_like(out), lse=torch.empty_like(lse))
    _check(out, lse, ref, ref_lse, dtype)
    # the general kernel
    lib.set_option(B.SMART_OPT_TVA_FORCE_GENERAL, 1)
    try:
        out, lse = call()
    finally:
        lib.set_option(B.SMART_OPT_TVA_FORCE_GENERAL, 0)
    _check(out, lse, ref, ref_lse, dtype)


@pytest.mark.parametrize("workers", [1, 3, 40])
def test_attention_cut_into_other_shares(lib, oracle_attention, workers):
    w = W.Workload("fp4", "bf16", 5, 8, 2, 128, 0, 0, seed=31)
    cu, parent = _trees([1, 6, 8, 30, 12])
    lens = np.array([900, 260, 1111, 333, 65], np.int32)
    call, scale, ref_args = _attend(lib, w, _case(w, cu, parent, lens, 16, 41), cu, parent, lens, 16)
    ref, ref_lse = oracle_attention.tree_attention(*ref_args, scale)
    lib.set_option(B.SMART_OPT_TVA_WORKERS, workers)
    try:
        out, lse = call()
    finally:
        lib.set_option(B.SMART_OPT_TVA_WORKERS, 0)
    _check(out, lse, ref, ref_lse, "bf16")


@pytest.mark.parametrize("workers,bs,heads", [(1, 16, (8, 2)), (9, 64, (8, 2)), (0, 24, (4, 1)), (5, 8, (7, 1)), (2, 16, (8, 1))])
def test_attention_of_many_rows_over_long_prefixes(lib, oracle_attention, workers, bs, heads):
    """Three and four row tiles of 32 rows over pieces of five and more steps of 128 keys, between pieces of fewer rows or steps."""
    import torch
    w = W.Workload("fp4", "bf16", 7, heads[0], heads[1], 128, 0, 0, seed=31)
    cu, parent = _trees([18, 3, 25, 32, 60, 128, 1])
    lens = np.array([900, 1030, 1337, 129, 641, 1500, 700], np.int32)
    call, scale, ref_args = _attend(lib, w, _case(w, cu, parent, lens, bs, 45), cu, parent, lens, bs)
    ref, ref_lse = oracle_attention.tree_attention(*ref_args, scale)
    lib.set_option(B.SMART_OPT_TVA_WORKERS, workers)
    try:
        out, lse = call()
        _check(out, lse, ref, ref_lse, "bf16")
        again = call()
    finally:
        lib.set_option(B.SMART_OPT_TVA_WORKERS, 0)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    out, lse = call(static=True, h_cu_nodes=cu, out=torch.empty_like(out), lse=torch.empty_like(lse))
    _check(out, lse, ref, ref_lse, "bf16")


@pytest.mark.parametrize("sizes", [[8] * 30, [2] * 29 + [128], [0, 3] * 15 + [9]])
def test_one_workgroup_a_segment_with_more_workgroups_than_compute_units(lib, oracle_attention, sizes):
    """30 sequences of 8 kv heads: the launch allows for more segments than there are; trees of one to four row groups."""
    import torch
    w = W.Workload("fp4", "bf16", len(sizes), 32, 8, 128, 0, 0, seed=31)
    cu, parent = _trees(sizes)
    lens = np.random.default_rng(3).integers(0, 200, len(sizes)).astype(np.int32)
    call, scale, ref_args = _attend(lib, w, _case(w, cu, parent, lens, 16, 49), cu, parent, lens, 16)
    ref, ref_lse = oracle_attention.tree_attention(*ref_args, scale)
    out, lse = call()
    _check(out, lse, ref, ref_lse, "bf16")
    again, again_lse = call(static=True, out=torch.empty_like(out), lse=torch.empty_like(lse))
    _check(again, again_lse, ref, ref_lse, "bf16")


def test_attention_on_a_cache_with_NaN_blocks_and_bad_table_entries(lib, oracle_attention):
    """A NaN key block makes its sequence's rows NaN, and nobody else's; a table entry outside the cache is reported."""
    import torch
    w = W.Workload("fp4", "bf16", 3, 8, 2, 128, 0, 0, seed=31)
    cu, parent = _trees([3, 2, 5])
    lens = np.array([100, 200, 90], np.int32)
    case = _case(w, cu, parent, lens, 16, 42)
    call, scale, ref_args = _attend(lib, w, case, cu, parent, lens, 16)
    ref, _ = oracle_attention.tree_attention(*ref_args, scale)
    table = case[3].cpu().numpy()
    case[1][int(table[1, 3]), 1, F.scale_at("k", 5, 40, 16, 128)] = 255
    out, _ = call()
    got = H.out_to_f64(out, "bf16")
    assert np.isnan(got[cu[1]:cu[2], 4:]).all()
    keep = np.ones_like(got, bool)
    keep[cu[1]:cu[2], 4:] = False
    assert H.rel_err(got[keep], ref[keep]) <= 2.0 ** -7
    case[3][0, 2] = 10 ** 6
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    call(status=status)
    assert status.tolist() == [B.SMART_TVA_BAD_BLOCK, 0, 0]


def test_attention_of_huge_values(lib, oracle_attention):
    """Stored values up to 6 2^125 and weights whose smaller parts would turn an infinite product into NaN."""
    w = W.Workload("fp4", "bf16", 2, 4, 1, 128, 0, 0, seed=31)
    cu, parent = _trees([2, 3])
    lens = np.array([70, 40], np.int32)
    case = _case(w, cu, parent, lens, 16, 43)
    values = case[4][4]
    table = case[3].cpu().numpy()
    for s in range(16):
        for j in range(4):
            case[2][int(table[0, 1]), 0, F.scale_at("v", s, 32 * j, 16, 128)] = 240
    values[int(table[0, 1])] = F.decode_pages(case[2].cpu().numpy(), "v", 16, 128)[int(table[0, 1])]
    call, scale, ref_args = _attend(lib, w, case, cu, parent, lens, 16)
    ref, ref_lse = oracle_attention.tree_attention(*ref_args, scale)
    out, lse = call()
    for b in range(2):
        _check(out[cu[b]:cu[b + 1]], lse[cu[b]:cu[b + 1]], ref[cu[b]:cu[b + 1]], ref_lse[cu[b]:cu[b + 1]], "bf16")


def test_capacity_rows_and_empty_batches(lib):
    import torch
    w = W.Workload("fp4", "bf16", 2, 8, 2, 128, 0, 0, seed=31)
    cu, parent = _trees([3, 2])
    lens = np.array([100, 0], np.int32)
    case = _case(w, cu, parent, lens, 16, 44)
    call, _, _ = _attend(lib, w, case, cu, parent, lens, 16)
    ref, ref_lse = call()
    args, kc, vc, table, _ = case
    pad = lambda t: torch.cat([t, torch.full((4,) + t.shape[1:], float("nan"), dtype=t.dtype, device="cuda")])
    mask = lib.tree_pack(_dev(cu), _dev(parent), _dev(lens))[3]
    mask = torch.cat([mask, torch.zeros((4, 2), dtype=torch.int64, device="cuda")])
    out, lse = lib.tree_verify_attention(*(pad(t) for t in args), kc, vc, table, _dev(lens), _dev(cu), mask, 128 ** -0.5,
                                         B.SMART_KV_INTERLEAVED, kv_cache_dtype=B.SMART_FP4_E2M1, want_lse=True)
    assert torch.equal(out[:5], ref) and torch.equal(lse[:5], ref_lse)
    none = lib.tree_verify_attention(*(t[:0] for t in args), kc, vc, table[:0], _dev(lens)[:0], _dev(cu)[:1] * 0, mask[:0], 0.1,
                                     B.SMART_KV_INTERLEAVED, kv_cache_dtype=B.SMART_FP4_E2M1)
    assert none.shape[0] == 0


@pytest.mark.parametrize("dtype,D,sizes,stride", [("bf16", 128, [3, 30], 1 << 29), ("f32", 64, [3, 30], 1 << 29), ("bf16", 128, [2, 3], 1 << 32)])
def test_pages_far_apart(lib, oracle_attention, dtype, D, sizes, stride):
    """Offsets past 32 bits: the blocks of a cache 2^29 bytes apart, and 2^32 (which the general kernel serves)."""
    import torch
    w = W.Workload("fp4", dtype, 2, 8, 2, D, 0, 0, seed=31)
    cu, parent = _trees(sizes)
    lens = np.array([[700, 90], [40, 3]][stride > 1 << 29], np.int32)
    bs = 64 if stride == 1 << 29 else 16
    args, kc, vc, table, ref_args = _case(w, cu, parent, lens, bs, 46)
    nb, heads, page = kc.shape
    store = torch.empty((nb - 1) * stride + 2 * heads * page, dtype=torch.uint8, device="cuda")
    far = [store.as_strided(kc.shape, (stride, page, 1), o) for o in (0, heads * page)]
    assert store.numel() > 1 << 32
    slots = _dev(np.arange(nb * bs).astype(np.int64))
    rows = lib.kv_cache_read_fp4(slots, kc, vc, D, bs, torch.float32)
    lib.kv_cache_write_fp4(*rows, slots, *far, bs)                    # (values of the format come out as they are)
    again = lib.kv_cache_read_fp4(slots, *far, D, bs, torch.float32)
    for a, b in zip(rows, again):
        assert torch.equal(a.view(torch.int32).masked_fill(a.isnan(), 0), b.view(torch.int32).masked_fill(b.isnan(), 0))
        assert torch.equal(a.isnan(), b.isnan())
    call, scale, _ = _attend(lib, w, (args, far[0], far[1], table, ref_args), cu, parent, lens, bs)
    ref, ref_lse = oracle_attention.tree_attention(*ref_args, scale)
    _check(*call(), ref, ref_lse, dtype)


def test_a_slot_named_twice(lib):
    """Holds codes and scales of the rows that named it; nothing else changes."""
    import torch
    bs, D = 8, 64
    k, _ = _rows(3, 1, D, "bf16", 11)
    v, _ = _rows(3, 1, D, "bf16", 12)
    kc, vc = (torch.full((2, 1, F.page_bytes(bs, D)), 0x77, dtype=torch.uint8, device="cuda") for _ in range(2))
    lib.kv_cache_write_fp4(k, v, _dev(np.array([9, 3, 9], np.int64)), kc, vc, bs)
    for c, i in ((kc, 0), (vc, 1)):
        alone = []
        for t in (0, 2):
            one = [torch.full_like(kc, 0x77) for _ in range(2)]
            lib.kv_cache_write_fp4(k[1:], v[1:], _dev(np.array([3, -1], np.int64)), *one, bs)
            lib.kv_cache_write_fp4(k[t:t + 1], v[t:t + 1], _dev(np.array([9], np.int64)), *one, bs)
            alone.append(one[i])
        assert ((c == alone[0]) | (c == alone[1])).all()


def test_calls_on_two_streams_at_once():
    import torch
    libs = B.SmartTree(0), B.SmartTree(0)                             # a workspace each
    w = W.Workload("fp4", "bf16", 5, 8, 2, 128, 0, 0, seed=31)
    cu, parent = _trees([1, 6, 33, 20, 12])
    lens = np.array([900, 2060, 1111, 1333, 65], np.int32)
    calls = [_attend(lib, w, _case(w, cu, parent, lens, 16, 47 + i), cu, parent, lens, 16)[0] for i, lib in enumerate(libs)]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        got = []
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                got.append([c() for _ in range(4)])
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            for x in a:
                assert torch.equal(x[0], b[0]) and torch.equal(x[1], b[1])


@pytest.mark.parametrize("dtype,D,bs", [("bf16", 128, 16), ("f32", 64, 24)])
def test_commit(lib, dtype, D, bs):
    import torch
    Hkv, sizes, depth = 2, [5, 9, 1, 12, 3], 4
    cu, parent = _trees(sizes, 3)
    k, k64 = _rows(int(cu[-1]), Hkv, D, dtype, 5)
    v, v64 = _rows(int(cu[-1]), Hkv, D, dtype, 6)
    lens = np.array([0, bs - 1, 3 * bs, bs + 3, 4 * bs - 1], np.int32)
    nb, room = 25, 4
    table = np.random.default_rng(7).permutation(nb)[:5 * room].reshape(5, room).astype(np.int32)
    path = np.full((5, depth + 1), -1, np.int32)
    accepted = np.array([2, 4, 0, 1, 1], np.int32)                  # the last one has no room
    for b, a in enumerate(accepted):
        path[b, :a + 1] = np.sort(np.random.default_rng(b).permutation(sizes[b])[:a + 1])
    path[3, 1] = sizes[3]                                           # no node of the tree
    page = F.page_bytes(bs, D)
    kc, vc = (torch.full((nb, Hkv, page), 0x33, dtype=torch.uint8, device="cuda") for _ in range(2))
    new, status = lib.tree_commit_fp4(_dev(cu), _dev(accepted), _dev(path), k, v, kc, vc, _dev(table), _dev(lens), bs)
    assert status.tolist() == [0, 0, 0, B.SMART_ETREE, B.SMART_ECAP]
    assert new.tolist() == [3, bs + 4, 3 * bs + 1, bs + 3, 4 * bs - 1]
    for which, c, x in (("k", kc, k64), ("v", vc, v64)):
        codes, scales = F.encode(x)
        pages = np.full((nb, Hkv, page), 0x33, np.uint8)
        for b in range(3):
            for i in range(accepted[b] + 1):
                at, node = lens[b] + i, cu[b] + path[b, i]
                for g in range(Hkv):
                    F.put_row(pages[table[b, at // bs], g], which, at % bs, codes[node, g], scales[node, g], bs)
        assert np.array_equal(c.cpu().numpy(), pages)


def test_prefill_then_steps_as_they_are_used(lib, oracle_attention):
    """Prompts through rope, prompt_attention and kv_cache_write_fp4; then trees over the 4-bit cache, committed, and trees again;
    the step captured in a graph gives the eager result on every replay."""
    import torch
    from oracle import prompt as P
    Hq, Hkv, D, bs = 8, 2, 128, 16
    lens = np.array([45, 7, 130], np.int32)
    cu_t = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T = int(cu_t[-1])
    g = torch.Generator().manual_seed(21)
    q, k, v = (torch.randn((T, h, D), generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    pos = _dev(np.concatenate([np.arange(m) for m in lens]), np.int32)
    lib.tree_rope(pos, q, k)
    out = lib.prompt_attention(q, k, v, _dev(cu_t), D ** -0.5)
    f = lambda t: t.double().cpu().numpy()
    ref = P.prompt_attention(f(q), f(k), f(v), cu_t, D ** -0.5)[0]
    assert H.rel_err(f(out), ref) <= 2.0 ** -7
    room = 10
    table = np.random.default_rng(3).permutation(3 * room).reshape(3, room).astype(np.int32)
    slots = np.concatenate([table[b, np.arange(m) // bs].astype(np.int64) * bs + np.arange(m) % bs for b, m in enumerate(lens)])
    kc, vc = (torch.zeros((3 * room, Hkv, B.fp4_page_bytes(bs, D)), dtype=torch.uint8, device="cuda") for _ in range(2))
    lib.kv_cache_write_fp4(k, v, _dev(slots), kc, vc, bs)
    cu, parent = _trees([4, 9, 2], 5)
    d_cu, d_par, d_table = _dev(cu), _dev(parent), _dev(table)
    token = _dev(np.arange(int(cu[-1])) % 7, np.int32)
    length = _dev(lens)
    lib.reserve(3, int(cu[-1]), Hq, Hkv)

    def step(length, q, kt, vt):
        _, position, _, mask, _ = lib.tree_pack(d_cu, d_par, length)
        out = lib.tree_verify_attention(q, kt, vt, kc, vc, d_table, length, d_cu, mask, D ** -0.5, B.SMART_KV_INTERLEAVED, block_size=bs,
                                        kv_cache_dtype=B.SMART_FP4_E2M1)
        accepted, path, _ = lib.tree_accept(d_cu, d_par, token, token.roll(-1), 4)
        new, status = lib.tree_commit_fp4(d_cu, accepted, path, kt, vt, kc, vc, d_table, length, bs)
        return out, new, status

    for i in range(3):
        qs, kt, vt = (torch.randn((int(cu[-1]), h, D), generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
        dec = [F.decode_pages(c.cpu().numpy(), w, bs, D) for w, c in (("k", kc), ("v", vc))]
        ref = oracle_attention.tree_attention(f(qs), f(kt), f(vt), *dec, table, length.cpu().numpy(), cu, parent, D ** -0.5)[0]
        out, new, status = step(length, qs, kt, vt)
        assert H.rel_err(f(out), ref) <= 2.0 ** -7 and not status.any() and (new > length).all()
        length = new.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(length, qs, kt, vt)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = step(length, qs, kt, vt)
    for i in range(4):
        qs.mul_(-0.5)
        want = [x.clone() for x in step(length, qs, kt, vt)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert H.rel_err(f(res[0]), f(want[0])) <= 2.0 ** -7 and torch.equal(res[1], want[1]) and torch.equal(res[2], want[2])
        (torch.ones(3, device="cuda") * i).sum().item()
