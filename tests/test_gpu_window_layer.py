"""The calls of a windowed layer together, as a server makes them: pages for prompts, norms and rotations, the cache written by the
slot map, attention of the prompts; then steps of pages given back and taken, a draft tree verified, its accepted path appended; in
between sequences end and others come.  Every output is compared with the definition over the whole history in binary64, bounds as in
test_gpu_tree_window.py."""
import numpy as np
import pytest

from oracle import prompt as P
from oracle import window as OW
from paper_2604_09731_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HQ, HKV, D, BS, WINDOW, SINKS, DEPTH = 4, 2, 64, 16, 40, 19, 5


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return B.SmartTree(0)


def _near(got, row, dtype):
    ref, _, A, S, n = row
    tol = (((2 * D + 2) * S + 2 * n + 32) * U) * A + (3 * 2.0 ** -8 * A if dtype == "bf16" else U * np.abs(ref))
    return (np.abs(got - ref) <= tol).all()


@pytest.mark.parametrize("dtype,layout", [("bf16", B.SMART_KV_INTERLEAVED), ("f32", B.SMART_KV_PLAIN)])
def test_a_server_of_one_layer(lib, dtype, layout):
    import torch
    rng, g = np.random.default_rng(7), torch.Generator().manual_seed(7)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    f = lambda x: x.double().cpu().numpy()
    rows, width, num_blocks = 6, 20, 45            # sequences, blocks of a table's row, pages: not enough without giving back
    shape = dict(zip(("k", "v"), ((num_blocks, HKV, D // 8, BS, 8), (num_blocks, HKV, BS // 8, D, 8)))) if layout == B.SMART_KV_INTERLEAVED else \
        dict(k=(num_blocks, HKV, BS, D), v=(num_blocks, HKV, BS, D))
    kc, vc = (torch.full(shape[x], float("nan"), dtype=dt, device="cuda") for x in "kv")
    strides = dict(block_size=BS, num_blocks=num_blocks, block_stride=HKV * BS * D, head_stride=BS * D, token_stride=D)
    weights = [(1 + 0.2 * torch.randn(D, generator=g)).to(dt).cuda() for _ in range(2)]
    table = torch.full((rows, width), -7, dtype=torch.int32, device="cuda")
    free, count = dev(rng.permutation(num_blocks).tolist()), dev([num_blocks])
    length, held, released = (dev([0] * rows) for _ in range(3))
    history = [(np.zeros((0, HKV, D)), np.zeros((0, HKV, D))) for _ in range(rows)]

    def project(positions):
        """Queries, keys and values of some tokens: parts of one projection's output, normed and rotated."""
        x = torch.randn((len(positions), (HQ + 2 * HKV) * D), generator=g).to(dt).cuda()
        q, k, v = (t.unflatten(1, (-1, D)) for t in x.split([HQ * D, HKV * D, HKV * D], 1))
        q, k = lib.tree_norm_rope(positions, q, k, *weights, base=500.0)
        return q, k, v.contiguous()

    def admit(lens):
        nonlocal length, held, count
        total = sum(lens)
        start = length
        cu, slots, length, held, count, status = lib.kv_cache_extend(length, dev(lens), held, table, free, count, BS, num_blocks, total + 9)
        assert not status.any() and cu.tolist() == np.concatenate([[0], np.cumsum(lens)]).tolist()
        position = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).cuda()
        q, k, v = project(position)
        lib.kv_cache_write(k, v, slots, kc, vc, layout, **strides)
        out = f(lib.prompt_attention(q, k, v, cu, D ** -0.5, window=WINDOW, sinks=SINKS))
        q, k, v = f(q), f(k), f(v)
        for b, n in enumerate(lens):
            if n == 0:
                continue
            lo = int(cu[b])
            history[b] = (k[lo:lo + n], v[lo:lo + n])
            for t in {0, n - 1, *rng.integers(0, n, 12).tolist()}:
                own = lo + np.array(P.seen(t, WINDOW, SINKS))
                for h in range(HQ):
                    assert _near(out[lo + t, h], (*P.prompt_row(q[lo + t, h], k[own, h // 2], v[own, h // 2], D ** -0.5), len(own)), dtype)

    def verify():
        nonlocal length, held, count
        _, _, _, held, count, status = lib.kv_cache_extend(length, dev([DEPTH + 1 if n else 0 for n in length.tolist()]), held, table, free,
                                                           count, BS, num_blocks, rows * (DEPTH + 1))
        assert not status.any()
        sizes = [int(rng.integers(1, 9)) if len(history[b][0]) else 0 for b in range(rows)]    # (none for rows without a sequence)
        cu = dev(np.concatenate([[0], np.cumsum(sizes)]).tolist())
        parent = dev([-1 if i == 0 else int(rng.integers(max(0, i - 3), i)) for n in sizes for i in range(n)])
        token = dev(rng.integers(0, 3, sum(sizes)).tolist())
        depth, position, _, mask, status = lib.tree_pack(cu, parent, length)
        assert status.tolist() == [0 if n else -2 for n in sizes]
        q, k, v = project(position)
        bad = torch.full((rows,), 9, dtype=torch.int32, device="cuda")
        out = f(lib.tree_verify_attention(q, k, v, kc, vc, table, length, cu, mask, D ** -0.5, layout, block_size=BS, status=bad, window=WINDOW,
                                          sinks=SINKS))
        assert not bad.any()
        fq, fk, fv, words, offsets = f(q), f(k), f(v), mask.cpu().numpy(), cu.tolist()
        for b in range(rows):
            lo, hi = offsets[b], offsets[b + 1]
            assert len(history[b][0]) == int(length[b])
            for i in range(lo, hi):
                line = OW.line_of(words[i], hi - lo)
                for h, row in enumerate(OW.node_rows(fq[i], fk[lo:hi], fv[lo:hi], line, *history[b], WINDOW, SINKS, D ** -0.5)):
                    assert _near(out[i, h], row, dtype), (b, i - lo, h)
        target = dev(rng.integers(0, 3, sum(sizes)).tolist())
        accept, path, _ = lib.tree_accept(cu, parent, token, target, DEPTH)
        live = length > 0
        new_length, status = lib.tree_commit(cu, accept, path, k, v, kc, vc, table, length, layout, **strides)
        for b in range(rows):
            if not live[b]:
                assert int(status[b]) == B.SMART_ETREE                         # nothing is appended
                continue
            assert int(status[b]) == 0
            new = [offsets[b] + j for j in path[b].tolist()[:int(accept[b]) + 1]]
            history[b] = tuple(np.concatenate([old, x[new]]) for old, x in zip(history[b], (fk, fv)))
        length = torch.where(live, new_length, length)

    def give_back(done):
        nonlocal length, held, released, count
        length, held, released, count, status = lib.kv_cache_release(length, held, released, table, free, count, BS, finished=dev(done),
                                                                     window=WINDOW, sinks=SINKS)
        assert not status.any()
        for b in range(rows):
            if done[b]:
                history[b] = (np.zeros((0, HKV, D)), np.zeros((0, HKV, D)))
        owned = [table[b, j].item() for b in range(rows) for j in range(int(held[b])) if j * BS < SINKS or j >= int(released[b])]
        assert sorted(owned + free[:int(count)].tolist()) == list(range(num_blocks))    # nobody shares a page, none is lost

    admit([37, 130, 0, 5, 64, 0])
    for step in range(60):
        give_back([0] * rows)
        verify()
        if step == 9:
            give_back([0, 1, 0, 0, 0, 0])           # one ends, two come
            admit_lens = [0, 90, 41, 0, 0, 0]
            before = [length.clone(), held.clone()]
            keep = [b for b in range(rows) if admit_lens[b] == 0]
            admit(admit_lens)
            assert length[keep].tolist() == before[0][keep].tolist()
    assert max(len(h[0]) for h in history) > 100 and int(released.max()) > 4
