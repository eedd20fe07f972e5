"""GPU: windows in the forms that only large calls take: prompts in row tiles of 256 rows, windows that hide nothing, and trees whose
finishing kernel gives each eight rows to one wavefront; and the block-table check of every form."""
import numpy as np
import pytest

from oracle import prompt as P
from oracle import window as OW
from paper_2604_09731_amd import binding as B
from tests.test_gpu_prompt_attention import _f64, _inputs
from tests.test_gpu_prompt_window import _check_rows, _cu
from tests.test_gpu_tree_window import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return B.SmartTree(0)


# ---- prompts --------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("want_lse", [False, True])
def test_prompts_in_tall_row_tiles(lib, D, want_lse):
    """64 / 8 heads: 2^18 rows and a window of more than 2^14 rows of a kv head, from which tiles of 256 rows (32 tokens) are taken."""
    lens, window, sinks, Hq = [4200, 1, 77], 2100, 70, 64
    cu, d_cu = _cu(lens)
    q, k, v = _inputs(int(cu[-1]), Hq, 8, D, "bf16", 53)
    got = lib.prompt_attention(q, k, v, d_cu, D ** -0.5, want_lse=want_lse, window=window, sinks=sinks)
    out, lse = (_f64(got[0]), _f64(got[1])) if want_lse else (_f64(got), None)
    assert np.isfinite(out).all()
    rng = np.random.default_rng(1)
    edge = {0, 1, 31, 32, 63, 64, sinks - 1, sinks, window - 1, window, window + sinks - 1, window + sinks, window + sinks + 1, window + sinks + 63,
            2175, 2176, 2207, 2208, 4159, 4160, 4191, 4192, 4199}       # window edges; first and last tokens of row tiles
    picks = sorted(edge | set(rng.integers(0, 4200, 30).tolist()))
    rows = [(0, t, h) for t in picks for h in sorted({0, Hq - 1, int(rng.integers(Hq))})]
    rows += [(1, 0, h) for h in (0, 7, 63)] + [(2, t, h) for t in (0, 31, 32, 69, 70, 76) for h in (0, 9, 63)]
    _check_rows(out, lse, _f64(q), _f64(k), _f64(v), cu, window, sinks, "bf16", rows)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_bad_values_in_tall_row_tiles(lib, D, bad):
    """A value that is no number, seen by a window's length of tokens, enters their rows only."""
    import torch
    T, window, sinks, at, Hq = 4200, 2100, 70, 1000, 64
    cu, d_cu = _cu([T])
    q, k, v = _inputs(T, Hq, 8, D, "bf16", 59)
    v2 = v.clone()
    v2[at, 3] = bad                                                     # of one kv head
    out, lse = lib.prompt_attention(q, k, v2, d_cu, D ** -0.5, want_lse=True, window=window, sinks=sinks)
    seeing = torch.zeros((T, Hq), dtype=torch.bool, device="cuda")
    seeing[at:at + window, 24:32] = True
    assert torch.equal(torch.isfinite(out).all(-1), ~seeing) and not torch.isfinite(out[seeing]).any()
    rows = [(0, t, h) for t in (at - 1, at + window, at + window + 1, at + window + 40) for h in (23, 24, 31, 32)]
    rows += [(0, t, h) for t in (at, at + 1, at + window - 1) for h in (23, 32)]
    _check_rows(_f64(out), _f64(lse), _f64(q), _f64(k), _f64(v), cu, window, sinks, "bf16", rows)


@pytest.mark.parametrize("T,Hq,Hkv", [(2048, 32, 8), (8192, 64, 64), (700, 4, 4)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_window_that_hides_nothing_is_none(lib, T, Hq, Hkv, dtype):
    import torch
    if dtype == "f32":
        T = min(T, 2048)
    _, d_cu = _cu([T])
    q, k, v = _inputs(T, Hq, Hkv, 64, dtype, 61)
    want, want_lse = lib.prompt_attention(q, k, v, d_cu, 0.125, want_lse=True)
    for window, sinks in ((T, 0), (T, 5), (T - 300, 300), (1, T - 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        out, lse = lib.prompt_attention(q, k, v, d_cu, 0.125, want_lse=True, window=window, sinks=sinks)
        assert torch.equal(out, want) and torch.equal(lse, want_lse), (window, sinks)


# ---- trees ----------------------------------------------------------------------------------------------------------------
FORMS = [("bf16", "same", "interleaved", 128), ("bf16", "same", "plain", 128), ("bf16", "fp8", "plain", 128), ("bf16", "fp4", "interleaved", 128),
         ("bf16", "same", "interleaved", 64), ("f32", "same", "plain", 128), ("f32", "same", "interleaved", 64)]


def _some(c, per_tree, seed):
    rng = np.random.default_rng(seed)
    nodes = set()
    for lo, hi in zip(c.h_cu[:-1].tolist(), c.h_cu[1:].tolist()):
        nodes |= {lo, hi - 1} | set(rng.integers(lo, hi, per_tree).tolist())
    return nodes


@pytest.mark.parametrize("dtype,cache,layout,D", FORMS)
def test_many_rows_of_wide_trees(lib, dtype, cache, layout, D):
    """More than 5120 rows, over prefixes that are shared out: an empty mask among them, and lse wanted or not."""
    import torch
    rng = np.random.default_rng(7)
    lens, sizes = rng.integers(100, 4000, 24).tolist(), rng.integers(4, 65, 24).tolist()
    assert sum(sizes) * 16 > 5120
    c = Case(lib, lens, sizes, 1024, 4, Hq=16, Hkv=4, D=D, dtype=dtype, cache=cache, layout=layout, seed=71)
    empty = int(c.h_cu[5]) + 1
    c.mask[empty] = 0
    out, lse = c.run(lib)
    c.check(out, lse, _some(c, 1, 1) | {empty})
    assert torch.equal(c.run(lib, want_lse=False), out)


@pytest.mark.parametrize("dtype,cache,layout,D", FORMS)
def test_many_rows_of_chains_deeper_than_the_window(lib, dtype, cache, layout, D):
    """Nodes that the window of those below them has left, and nodes among the first tokens, in trees behind long stretches of them."""
    lens = [995, 1000, 990, 1500, 2300, 1061, 1100, 940]
    c = Case(lib, lens, [128, 100, 90, 128, 64, 65, 127, 1], 60, 1000, Hq=16, Hkv=4, D=D, dtype=dtype, cache=cache, layout=layout, seed=73, chain=True)
    assert int(c.h_cu[-1]) * 16 > 5120
    out, lse = c.run(lib)
    nodes = _some(c, 2, 2)
    for lo, hi in zip(c.h_cu[:-1].tolist(), c.h_cu[1:].tolist()):
        nodes |= {lo + i for i in (58, 59, 60, 61, 63, 64) if lo + i < hi}
    c.check(out, lse, nodes)


@pytest.mark.parametrize("dtype,layout,D", [("bf16", "interleaved", 128), ("bf16", "plain", 128), ("bf16", "interleaved", 64), ("f32", "plain", 128)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_bad_values_among_many_rows(lib, dtype, layout, D, bad):
    """A cached value that is no number, which the first eleven nodes of a chain see, enters their rows and no others."""
    import torch
    rng = np.random.default_rng(9)
    lens, sizes = rng.integers(300, 900, 24).tolist(), rng.integers(16, 40, 24).tolist()
    lens[2], sizes[2] = 2003, 20
    c = Case(lib, lens, sizes, 400, 700, Hq=16, Hkv=4, D=D, dtype=dtype, layout=layout, seed=79, chain=True)
    assert sum(sizes) * 16 > 5120
    lo, token = int(c.h_cu[2]), 2003 - 400 + 11
    page, slot = int(c.h_table[2, token // 16]), token % 16
    (c.vc[page, 1, slot] if layout == "plain" else c.vc[page, 1, slot // 8, :, slot % 8]).fill_(bad)
    out, lse = c.run(lib)
    seeing = torch.zeros(out.shape[:2], dtype=torch.bool, device="cuda")
    seeing[lo:lo + 11, 4:8] = True
    assert torch.equal(torch.isfinite(out).all(-1), ~seeing) and not torch.isfinite(out[seeing]).any() and torch.isfinite(lse).all()
    c.check(out, lse, set(range(lo + 11, lo + 20)) | {lo - 1, lo + 20})


@pytest.mark.parametrize("form", ["direct", "split", "many rows", "general"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_block_table_check_of_every_form(lib, form, dtype):
    """Entries of blocks with first tokens or tokens of the window are checked, at the edges of both, the others are not."""
    import torch
    if form == "direct":
        c = Case(lib, [500, 300], [3, 2], 100, 20, dtype=dtype, seed=4)
        edges = ((0, 1), (1, 1), (2, 0), (24, 0), (25, 1), (31, 1), (32, 0))
    elif form == "general":
        c = Case(lib, [500, 300], [3, 2], 100, 33, dtype=dtype, seed=4)
        edges = ((0, 1), (2, 1), (3, 0), (24, 0), (25, 1), (31, 1), (32, 0))
    else:                                                               # blocks 0 .. 62 and (5000 - 1100 + 1) / 16 = 243 ..
        many = form == "many rows"
        c = Case(lib, [5000, 3900] + [1200] * 22 * many, [3, 2] + [60] * 22 * many, 1100, 1000, Hq=4, Hkv=1, dtype=dtype, seed=4)
        assert (int(c.h_cu[-1]) * 4 > 5120) == many
        edges = ((0, 1), (62, 1), (63, 0), (242, 0), (243, 1), (312, 1), (313, 0))
    status = torch.full((len(c.lens),), 7, dtype=torch.int32, device="cuda")
    clean = [0] * len(c.lens)
    lib.set_option(B.SMART_OPT_TVA_FORCE_GENERAL, int(form == "general"))
    try:
        c.run(lib, status=status)
        assert status.tolist() == clean
        for entry, bad in edges:
            for value in (-1, len(c.kc)):
                old = int(c.table[0, entry])
                c.table[0, entry] = value
                status.fill_(7)
                c.run(lib, status=status)
                assert status.tolist() == [bad] + clean[1:], (entry, value)
                c.table[0, entry] = old
    finally:
        lib.set_option(B.SMART_OPT_TVA_FORCE_GENERAL, 0)
