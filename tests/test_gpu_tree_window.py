"""GPU parity of tree_verify_attention with a window with the binary64 oracle.

Bounds per element, from what the kernels round (A = the row's softmax average of |v|, S = its largest scale * sum |q| |k|, n its
keys, u = 2^-24): scores 2 D u S in a weight's exponent, numerator and denominator, an fp8 cache's scale 2 u S more; sums of n
weights and of n weighted values 2 n u; exponentials, references, the merges of partial results and the division 32 u.  bf16 calls
round their weights to bf16 (2 2^-8 A, as a value and in the sum that divides), the general kernel does not; a bf16 result is
rounded by 2^-8 of itself.  Pages that nobody sees hold NaN, their entries of the table anything."""
import numpy as np
import pytest

from oracle import window as OW
from paper_2604_09731_amd import binding as B
from paper_2604_09731_amd import workloads as W

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
KS, VS = 0.0625, 0.03125


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return B.SmartTree(0)


def _trees(sizes, rng, chain):
    out = []
    for n in sizes:
        out.append([-1] * (n > 0) + [i - 1 if chain else int(rng.integers(max(0, i - 5), i)) for i in range(1, n)])
    return np.concatenate([np.array(t, np.int32) for t in out]) if out else np.zeros(0, np.int32)


class Case:
    """Inputs on the GPU, and the prefixes in float64."""

    def __init__(self, lib, lens, sizes, window, sinks, Hq=4, Hkv=2, D=64, bs=16, dtype="bf16", cache="same", layout="interleaved",
                 seed=0, chain=False):
        import torch
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.dtype, self.cache, self.window, self.sinks, self.bs, self.lens, self.scale = dtype, cache, window, sinks, bs, lens, D ** -0.5
        self.layout = B.SMART_KV_PLAIN if layout == "plain" else B.SMART_KV_INTERLEAVED
        self.h_cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
        N = int(self.h_cu[-1])
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        rand = lambda *s: torch.randn(s, generator=g)
        self.q, self.kt, self.vt = (rand(N, H, D).to(self.dt).cuda() for H in (Hq, Hkv, Hkv))
        self.parent = _trees(sizes, rng, chain)
        self.cu, self.len = t(self.h_cu), t(np.array(lens, np.int32))
        self.mask = lib.tree_pack(self.cu, t(self.parent), self.len)[3]
        # pages: those that somebody sees, a few spare ones that hold NaN
        live = [sorted({x // bs for x in OW.seen_tokens(n, n, window, sinks)}) for n in lens]
        nb = sum(map(len, live)) + 4
        perm, at = rng.permutation(nb), 0
        table = rng.integers(-9, nb + 9, (len(lens), max(1, (max(lens, default=0) + bs - 1) // bs + 1))).astype(np.int32)
        for b, pages in enumerate(live):
            table[b, pages] = perm[at:at + len(pages)]
            at += len(pages)
        k, v = rand(nb, Hkv, bs, D) * 1.5, rand(nb, Hkv, bs, D)
        spare = torch.from_numpy(perm[at:].copy())
        if cache == "fp4":
            kc, vc = (torch.zeros((nb, Hkv, -(-B.fp4_page_bytes(bs, D) // 16) * 16), dtype=torch.uint8, device="cuda") for _ in range(2))
            slots = torch.arange(nb * bs, device="cuda")
            k[spare], v[spare] = float("nan"), float("nan")
            rows = [x.transpose(1, 2).reshape(nb * bs, Hkv, D).contiguous().cuda() for x in (k, v)]
            lib.kv_cache_write_fp4(*rows, slots, kc, vc, bs)
            k, v = (x.view(nb, bs, Hkv, D).transpose(1, 2).cpu() for x in lib.kv_cache_read_fp4(slots, kc, vc, D, bs, torch.float32))
        else:
            if cache == "fp8":
                kc, vc = ((x / s).to(torch.float8_e4m3fn) for x, s in ((k, KS), (v, VS)))
                k, v = kc.double() * KS, vc.double() * VS
                kc, vc = kc.view(torch.uint8), vc.view(torch.uint8)
                kc[spare], vc[spare] = 0x7F, 0x7F
            else:
                kc, vc = k.to(self.dt), v.to(self.dt)
                k, v = kc.double(), vc.double()
                kc[spare], vc[spare] = float("nan"), float("nan")
            kc, vc = kc.cuda(), vc.cuda()
            if layout == "interleaved":
                kc, vc = B.interleave_kv_cache(kc, vc)
        self.kc, self.vc, self.table, self.h_table, self.k64, self.v64 = kc, vc, t(table), table, k.double().numpy(), v.double().numpy()

    def run(self, lib, want_lse=True, **kw):
        more = dict(kv_cache_dtype=B.SMART_FP4_E2M1) if self.cache == "fp4" else dict(k_scale=KS, v_scale=VS) if self.cache == "fp8" else {}
        return lib.tree_verify_attention(self.q, self.kt, self.vt, self.kc, self.vc, self.table, self.len, self.cu, self.mask, self.scale,
                                         self.layout, block_size=self.bs, want_lse=want_lse, window=self.window, sinks=self.sinks, **more, **kw)

    def prefix(self, b):
        n, (nb, H, bs, D) = self.lens[b], self.k64.shape
        t = np.arange(n)
        page = np.clip(self.h_table[b, t // bs], 0, nb - 1)
        return self.k64[page, :, t % bs], self.v64[page, :, t % bs]

    def check(self, out, lse, nodes=None, rounded=True):
        f = lambda x: x.double().cpu().numpy()
        got, got_lse, q, kt, vt, words = f(out), None if lse is None else f(lse), f(self.q), f(self.kt), f(self.vt), self.mask.cpu().numpy()
        D = q.shape[2]
        for b in range(len(self.lens)):
            lo, hi = int(self.h_cu[b]), int(self.h_cu[b + 1])
            if lo == hi:
                continue
            kp, vp = self.prefix(b)
            for i in range(lo, hi):
                if nodes is not None and i not in nodes:
                    continue
                rows = OW.node_rows(q[i], kt[lo:hi], vt[lo:hi], OW.line_of(words[i], hi - lo), kp, vp, self.window, self.sinks, self.scale)
                for h, (ref, ref_lse, A, S, n) in enumerate(rows):
                    u = ((2 * D + 2) * S + 2 * n + 32) * U
                    tol = u * A + (2.0 ** -8 if self.dtype == "bf16" else U) * np.abs(ref)
                    if self.dtype == "bf16" and rounded:
                        tol = tol + 2 * 2.0 ** -8 * A
                    err = np.abs(got[i, h] - ref)
                    assert (err <= tol).all(), (b, i - lo, h, np.max(err / np.maximum(tol, 1e-300)))
                    if got_lse is not None:
                        assert got_lse[i, h] == ref_lse or abs(got_lse[i, h] - ref_lse) <= u + 2 * U * abs(ref_lse), (b, i - lo, h)


KINDS = [("bf16", "same", "interleaved"), ("bf16", "same", "plain"), ("f32", "same", "interleaved"), ("f32", "same", "plain"),
         ("bf16", "fp8", "interleaved"), ("bf16", "fp8", "plain"), ("f32", "fp8", "plain"), ("f32", "fp8", "interleaved"),
         ("bf16", "fp4", "interleaved"), ("f32", "fp4", "interleaved")]


@pytest.mark.parametrize("dtype,cache,layout", KINDS)
@pytest.mark.parametrize("D,bs", [(128, 16), (64, 16), (64, 32), (128, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 2), (9, 0), (17, 30), (64, 4), (100, 65)])
def test_short_prefixes(lib, dtype, cache, layout, D, bs, window, sinks):
    c = Case(lib, [0, 1, 8, 57, 130, 200], [5, 1, 0, 12, 9, 3], window, sinks, D=D, bs=bs, dtype=dtype, cache=cache, layout=layout,
             seed=window + sinks)
    c.check(*c.run(lib))


@pytest.mark.parametrize("dtype,cache,layout", KINDS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 3), (40, 0), (126, 20), (200, 400)])
def test_chains_deeper_than_the_window(lib, dtype, cache, layout, window, sinks):
    c = Case(lib, [30, 0, 300], [128, 90, 65], window, sinks, Hq=2, Hkv=2, dtype=dtype, cache=cache, layout=layout, chain=True, seed=3)
    out, lse = c.run(lib)
    nodes = set(range(0, 283, 7)) | {0, 63, 64, 127, 128, 217, 218, 282}
    c.check(out, lse, nodes)


@pytest.mark.parametrize("dtype,cache,layout", KINDS)
@pytest.mark.parametrize("D,Hq,Hkv,sizes", [(128, 8, 2, [7, 20, 1, 33]), (64, 28, 4, [10, 3, 64, 2])])
def test_long_prefixes_split_and_workspace_free(lib, dtype, cache, layout, D, Hq, Hkv, sizes):
    """Long enough for shares that end anywhere; the same call captured takes the workspace-free form."""
    import torch
    c = Case(lib, [3001, 1500, 700, 2222], sizes, 1111, 13, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, cache=cache, layout=layout, seed=11)
    nodes = {int(n) for n in c.h_cu[:-1]} | {int(n) - 1 for n in c.h_cu[1:]} | {9, 25}
    out, lse = c.run(lib)
    c.check(out, lse, nodes)
    out2, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.run(lib, out=out2, lse=lse2)
    for _ in range(3):
        out2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        c.check(out2, lse2, nodes)
        again, _ = c.run(lib)
        assert torch.equal(again, out)
    bare = c.run(lib, want_lse=False)
    assert torch.equal(bare, out)


@pytest.mark.parametrize("dtype,cache,layout", KINDS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 3), (50, 4), (130, 70)])
def test_general_kernel(lib, dtype, cache, layout, window, sinks):
    c = Case(lib, [0, 1, 57, 300, 130], [5, 1, 70, 12, 0], window, sinks, dtype=dtype, cache=cache, layout=layout, seed=5, chain=window == 2)
    lib.set_option(B.SMART_OPT_TVA_FORCE_GENERAL, 1)
    try:
        out, lse = c.run(lib)
    finally:
        lib.set_option(B.SMART_OPT_TVA_FORCE_GENERAL, 0)
    c.check(out, lse, set(range(0, 88, 5)) | {5, 75, 87}, rounded=False)


@pytest.mark.parametrize("dtype,cache,layout", [KINDS[0], KINDS[3], KINDS[8]])
@pytest.mark.parametrize("window", [400, 2 ** 31 - 1])
def test_windows_that_hide_nothing(lib, dtype, cache, layout, window):
    import torch
    c = Case(lib, [100, 3, 256], [4, 17, 9], window, 2 ** 31 - 1, D=128, dtype=dtype, cache=cache, layout=layout, seed=2)
    out, lse = c.run(lib)
    c.check(out, lse)
    c.window, c.sinks = None, 0
    if window > 1000:
        assert torch.equal(c.run(lib)[0], out)


def test_a_few_tokens_at_the_end_of_a_long_table(lib):
    """Many sequences, far pages, windows that end anywhere in a page, one block size of 8 tokens and one of 24."""
    for bs, layout in ((8, "interleaved"), (24, "interleaved"), (24, "plain"), (40, "plain")):
        lens = [2000 + 7 * i for i in range(20)] + [0, 33, 34, 35]
        c = Case(lib, lens, [1 + i % 4 for i in range(24)], 34, 11, Hq=2, Hkv=1, D=128, bs=bs, layout=layout, seed=bs)
        c.check(*c.run(lib))


@pytest.mark.parametrize("dtype,cache", [("bf16", "same"), ("f32", "same"), ("bf16", "fp8"), ("bf16", "fp4")])
def test_bad_values_behind_the_window_and_inside_it(lib, dtype, cache):
    """An infinity or NaN in a page that nobody may see a token of, but that holds the window's first one, enters nobody's row; one
    that some nodes see makes their rows what the formula gives."""
    import torch
    c = Case(lib, [205, 120], [9, 6], 60, 3, D=64, dtype=dtype, cache=cache, layout="plain" if cache == "same" else "interleaved", seed=8, chain=True)
    ref, ref_lse = c.run(lib)
    b, first = 0, 205 - 60 + 1                  # the root sees tokens 146 .. 204, the node below it 147 ..
    for token, seen_by in ((145, 0), (147, 2), (4, 0), (200, 9)):
        page, slot = int(c.h_table[b, token // 16]), token % 16
        kc, vc = c.kc.clone(), c.vc.clone()
        if cache == "fp4":
            slots = torch.tensor([page * 16 + slot], device="cuda")
            k, v = lib.kv_cache_read_fp4(slots, c.kc, c.vc, 64, 16)
            lib.kv_cache_write_fp4(k, torch.full_like(v, float("nan")), slots, c.kc, c.vc, 16)
        elif cache == "fp8":
            c.vc[page, :, slot // 8, :, slot % 8] = 0x7F
        else:
            c.vc[page, :, slot] = float("inf")
        out, lse = c.run(lib)
        assert torch.isfinite(lse).all()
        good = [i for i in range(15) if i >= seen_by or i >= 9]
        near = 2.0 ** -6 if dtype == "bf16" else 1e-5
        assert (out[good].float() - ref[good].float()).abs().max() <= near * ref.float().abs().max(), token
        assert not torch.isfinite(out[:min(seen_by, 9)]).any(), token
        c.kc.copy_(kc)
        c.vc.copy_(vc)


def test_status_looks_at_what_is_read(lib):
    import torch
    c = Case(lib, [500, 300], [3, 2], 100, 20, seed=4)
    status = torch.full((2,), 7, dtype=torch.int32, device="cuda")
    for want_split in (True, False):
        c.run(lib, status=status)
        assert status.tolist() == [0, 0]
    for entry, bad in ((0, 1), (1, 1), (2, 0), (24, 0), (25, 1), (31, 1), (32, 0)):
        old = int(c.table[0, entry])
        c.table[0, entry] = -1
        c.run(lib, status=status)
        assert status.tolist() == [bad, 0], entry
        c.table[0, entry] = old


def test_offsets_that_are_no_running_sum(lib):
    """Rows are given to the sequence that a search finds, as without a window."""
    import torch
    for dtype in ("bf16", "f32"):
        c = Case(lib, [200, 100, 50], [4, 5, 6], 60, 2, dtype=dtype, layout="plain", seed=6)
        for cu in ([0, 9, 4, 15], [2, 4, 9, 12], [0, 4, 9, 99], [-3, 4, 9, 15]):
            c.cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
            out, lse = c.run(lib)
            lib.set_option(B.SMART_OPT_TVA_FORCE_GENERAL, 1)
            want, want_lse = c.run(lib)
            lib.set_option(B.SMART_OPT_TVA_FORCE_GENERAL, 0)
            assert (out.float() - want.float()).abs().max() <= (2.0 ** -7 if dtype == "bf16" else 1e-5) * 4
            assert torch.equal(lse.isinf(), want_lse.isinf()) and (lse - want_lse)[~lse.isinf()].abs().max() <= 1e-4


def test_rows_that_are_not_aligned(lib):
    """Tensors off 16 bytes take the general kernel, and so does a call without a cache."""
    import torch
    c = Case(lib, [150, 20], [6, 3], 40, 5, dtype="f32", layout="plain", seed=9)
    wide = torch.zeros(c.q.numel() + 1, device="cuda")
    q = wide[1:].view(c.q.shape)
    q.copy_(c.q)
    c.q = q
    c.check(*c.run(lib))
    out = lib.tree_verify_attention(c.q, c.kt, c.vt, None, None, None, torch.zeros_like(c.len), c.cu, c.mask, c.scale, c.layout, window=2, sinks=1)
    c.lens, c.window, c.sinks = [0, 0], 2, 1
    c.check(out, None)


def test_nodes_behind_the_trees_and_empty_masks(lib):
    import torch
    c = Case(lib, [90, 40], [5, 4], 30, 2, D=128, seed=10)
    c.mask[3] = 0                                   # at its sequence's next position, without itself
    out, lse = c.run(lib)
    c.check(out, lse)
    c.mask[3] = 1 << 40                             # a bit behind the tree is none
    out2, lse2 = c.run(lib)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    c.window, c.sinks = 1, 0
    c.lens, c.len = [0, 40], torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    out, lse = c.run(lib)
    assert not out[3].any() and (lse[3] == float("-inf")).all()


def test_another_stream(lib):
    import torch
    c = Case(lib, [900, 350], [6, 8], 200, 4, D=128, seed=12)
    want = c.run(lib, want_lse=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.run(lib, want_lse=False)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype,cache,layout", [("bf16", "same", "interleaved"), ("f32", "same", "plain"), ("bf16", "fp8", "plain")])
def test_far_pages(lib, dtype, cache, layout):
    """Pages whose offsets pass 32 bits, in a cache of more than 4 GiB."""
    import torch
    c = Case(lib, [400, 90], [6, 4], 150, 20, D=128, dtype=dtype, cache=cache, layout=layout, seed=21)
    page = c.kc[0].numel()
    nb, first = (5 << 30) // (page * c.kc.element_size()), len(c.kc)
    far = []
    for x in (c.kc, c.vc):
        big = torch.empty((nb, *x.shape[1:]), dtype=x.dtype, device="cuda")
        big[nb - first:] = x
        far.append(big)
    c.kc, c.vc = far
    inside = (c.table >= 0) & (c.table < first)
    c.table = torch.where(inside, c.table + (nb - first), torch.full_like(c.table, -1))
    out, lse = c.run(lib)
    c.check(out, lse)                       # (the prefixes are those of the near pages)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch", [20, 200])
def test_windows_of_one_behind_full_tables(lib, dtype, batch):
    """Single tokens that see themselves only: every row is its own value, an infinity too; the table has no entry behind the prefix."""
    import torch
    c = Case(lib, [59 + 5 * (b % 2) for b in range(batch)], [1] * batch, 1, 0, dtype=dtype, seed=batch)
    c.table = c.table[:, :4].contiguous()
    c.vt[batch // 2:, :, 5] = float("inf")
    out, lse = c.run(lib)
    assert torch.equal(out, c.vt.repeat_interleave(2, 1))
    own = (c.q.double() * c.kt.double().repeat_interleave(2, 1)).sum(-1) * c.scale
    S = (c.q.double() * c.kt.double().repeat_interleave(2, 1)).abs().sum(-1).max().item() * c.scale
    assert (lse.double() - own).abs().max() <= ((2 * 64 + 2) * S + 34) * U + 2 * U * S
