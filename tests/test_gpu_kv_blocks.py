"""kv_cache_extend and kv_cache_release against the oracle that goes through the sequences one by one; everything is equal."""
import random

import pytest

from oracle import kv_blocks as K
from paper_2604_09731_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return B.SmartTree(0)


def _dev(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _extend(lib, length, new, held, table, free, count, bs, nb, cap):
    d = [_dev(x) for x in (length, new, held)]
    t, f = _dev(table).view(len(length), -1), _dev(free)
    got = lib.kv_cache_extend(*d, t, f, _dev([count]), bs, nb, cap)
    want = K.extend(length, new, held, table, free, count, bs, nb, cap)
    cu, slots, new_length, new_held, new_count, status = (x.tolist() for x in got)
    assert (cu, slots, new_length, new_held, new_count, status) == (want[0], want[1], want[2], want[3], [want[4]], want[5])
    assert t.tolist() == table and f.tolist() == free
    return want


def _release(lib, length, held, released, finished, table, free, count, bs, window, sinks):
    d = [_dev(x) for x in (length, held, released)]
    t, f = _dev(table).view(len(length), -1), _dev(free)
    got = lib.kv_cache_release(*d, t, f, _dev([count]), bs, finished=_dev([int(x) for x in finished]), window=window, sinks=sinks)
    want = K.release(length, held, released, finished, table, free, count, bs, window, sinks)
    assert [x.tolist() for x in got] == [want[0], want[1], want[2], [want[3]], want[4]]
    assert t.tolist() == table and f.tolist() == free
    return want


@pytest.mark.parametrize("seed", range(8))
def test_many_steps_of_a_server(lib, seed):
    rng = random.Random(seed)
    bs, n = rng.choice([1, 8, 16, 24, 64]), rng.choice([1, 2, 5, 40, 255, 256, 257, 700])
    width, window, sinks = rng.randrange(1, 30), *rng.choice([(0, 0), (1, 0), (40, 3), (100, 65)])
    nb = max(1, n * width // rng.choice([1, 2, 8]))
    table, free, count = [[-1] * width for _ in range(n)], list(range(nb)), nb
    rng.shuffle(free)
    length, held, released = [0] * n, [0] * n, [0] * n
    for step in range(8):
        new = [rng.choice([0, 1, 1, 9, bs, 3 * bs + 1]) for _ in range(n)]
        cap = max(0, sum(new) + rng.choice([0, 0, 100, -7]))
        _, _, length, held, count, status = _extend(lib, length, new, held, table, free, count, bs, nb, cap)
        done = [rng.random() < 0.15 for _ in range(n)]
        length, held, released, count, status = _release(lib, length, held, released, done, table, free, count, bs, window, sinks)


def test_one_long_prompt_and_capacity_rows(lib):
    free = list(range(9000))
    random.Random(0).shuffle(free)
    _extend(lib, [0, 5], [131072, 4], [0, 1], [[-1] * 8192, [8999] + [-1] * 8191], free, 8900, 16, 9000, 140000)
    _extend(lib, [131000], [80], [8190], [list(range(8190)) + [-1] * 10], free, 9000, 16, 9000, 80)


@pytest.mark.parametrize("length,new,held", [(-1, 3, 1), (3, -1, 1), (3, 1, -1), (3, 1, 6), (9, 1, 1), (2 ** 31 - 1, 2 ** 31 - 1, 5), (0, 2 ** 31 - 1, 0), (40, 1, 5), (40, 0, 5)])
def test_numbers_that_do_not_fit(lib, length, new, held):
    table = [[1, 2, -1, -1, -1], [3, 4, 5, 6, 7], [-1] * 5]
    want = _extend(lib, [5, length, 0], [4, new, 8], [1, held, 0], table, [9, 8, 10, 11], 4, 8, 20, 30)
    assert want[5][0] == K.OK
    _release(lib, [5, length, 0], [1, held, 0], [0, 0, 0], [False, True, False], table, [9] * 6, 1, 8, 2, 0)
    _release(lib, [5, length, 0], [1, held, 0], [0, max(0, held) + 1, 0], [False, True, False], table, [9] * 6, 1, 8, 2, 0)


def test_nothing_asked_behind_the_last_row(lib):
    want = _extend(lib, [3, 4, 5, 8], [4, 9, 0, 1], [1, 1, 1, 1], [[1, -1, -1], [2, -1, -1], [3, -1, -1], [4, -1, -1]], [0, 5], 2, 8, 6, 6)
    assert want[5] == [K.OK, K.ECAP, K.OK, K.ECAP]


@pytest.mark.parametrize("count", [-5, 0, 1, 2, 3, 4, 99])
def test_a_list_that_runs_short_or_over(lib, count):
    want = _extend(lib, [0, 8, 7, 0], [9, 0, 1, 1], [0, 1, 1, 0], [[-1] * 3, [4, -1, -1], [5, -1, -1], [-1] * 3], [0, 1, 2, 3], count, 8, 6, 11)
    assert want[5][1] == want[5][2] == K.OK                     # those that need none are served
    _release(lib, [24, 24, 3, 0], [3, 3, 1, 0], [0, 0, 0, 0], [True, False, True, True], [[1, 2, 3], [4, 5, 6], [7, 0, 0], [0] * 3], [0] * 4, count, 8, 9, 1)


def test_blocks_outside_the_cache_get_no_slots(lib):
    _extend(lib, [4, 8], [8, 16], [1, 1], [[-3, -1, -1], [2, -1, -1]], [1, 77, -9], 3, 8, 4, 24)


def test_empty_batches_and_no_rows(lib):
    import torch
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    cu, slots, length, held, count, status = lib.kv_cache_extend(e, e, e, torch.empty((0, 4), dtype=torch.int32, device="cuda"), _dev([1, 2]), _dev([2]), 16, 8, 5)
    assert cu.tolist() == [0] and slots.tolist() == [-1] * 5 and count.tolist() == [2] and length.numel() == 0
    assert lib.kv_cache_release(e, e, e, torch.empty((0, 4), dtype=torch.int32, device="cuda"), _dev([1, 2]), _dev([2]), 16)[3].tolist() == [2]
    _extend(lib, [3, 0], [0, 0], [1, 0], [[1, -1], [-1, -1]], [2], 1, 8, 4, 0)
    _extend(lib, [0, 0], [0, 3], [0, 0], [[], []], [2], 1, 8, 4, 3)
    _extend(lib, [0], [3], [0], [[-1]], [], 1, 8, 4, 3)


def test_without_finished_sequences_or_window(lib):
    length, held, zero, table, free = _dev([90]), _dev([6]), _dev([0]), _dev([[1, 2, 3, 4, 5, 6]]), _dev([0] * 6)
    assert [x.tolist() for x in lib.kv_cache_release(length, held, zero, table, free, zero, 16)] == [[90], [6], [0], [0], [0]]
    assert [x.tolist() for x in lib.kv_cache_release(length, held, zero, table, free, zero, 16, window=40, sinks=20)] == [[90], [6], [3], [1], [0]]
    assert free.tolist() == [3, 0, 0, 0, 0, 0]                  # blocks 0 and 1 hold the sinks, position 90 sees 51 ..


def test_captured_steps(lib):
    """A step of a captured decoding loop, replayed: releases, extends, and takes over the new numbers."""
    import torch
    n, bs, width, nb = 300, 16, 40, 6000
    state = [_dev([0] * n) for _ in range(3)]
    table, free, count, new = _dev([[-1] * width] * n), _dev(list(range(nb))), _dev([nb]), _dev([5 + i % 3 for i in range(n)])
    slots_out = torch.zeros(n * 8, dtype=torch.int64, device="cuda")

    def step():
        length, held, released, c, _ = lib.kv_cache_release(*state, table, free, count, bs, window=64, sinks=4)
        _, slots, length, held, c, _ = lib.kv_cache_extend(length, new, held, table, free, c, bs, nb, n * 8)
        for old, now in zip((*state, count, slots_out), (length, held, released, c, slots)):
            old.copy_(now)

    h = [[0] * n for _ in range(3)]
    h_table, h_free, h_count, h_new = [[-1] * width for _ in range(n)], list(range(nb)), nb, new.tolist()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    saved = [x.clone() for x in (*state, table, free, count)]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        step()
    for x, y in zip((*state, table, free, count), saved):
        x.copy_(y)
    for i in range(30):
        graph.replay()
        torch.cuda.synchronize()
        h[0], h[1], h[2], h_count, _ = K.release(h[0], h[1], h[2], [False] * n, h_table, h_free, h_count, bs, 64, 4)
        _, h_slots, h[0], h[1], h_count, _ = K.extend(h[0], h_new, h[1], h_table, h_free, h_count, bs, nb, n * 8)
        assert [x.tolist() for x in state] == h and count.item() == h_count and slots_out.tolist() == h_slots
        assert table.tolist() == h_table and free.tolist() == h_free
