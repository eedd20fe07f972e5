"""The block-table oracle by what has to hold whatever it does: nobody shares a page, none is lost, and windows keep what they see."""
import random

from oracle import kv_blocks as K


def test_pages_are_never_shared_or_lost():
    rng = random.Random(1)
    for trial in range(40):
        bs, B, width, nb = rng.choice([1, 8, 16]), rng.randrange(1, 7), rng.randrange(1, 12), rng.randrange(1, 40)
        window, sinks = rng.choice([(0, 0), (5, 0), (20, 3), (30, 17)])
        table, free, count = [[-1] * width for _ in range(B)], list(range(nb)), nb
        length, held, released = [0] * B, [0] * B, [0] * B
        for step in range(30):
            new = [rng.choice([0, 1, 3, bs, 2 * bs + 1]) for _ in range(B)]
            cap = rng.choice([sum(new), sum(new) + 5, max(0, sum(new) - 3)])
            cu, slots, length2, held, count, status = K.extend(length, new, held, table, free, count, bs, nb, cap)
            for b in range(B):
                if status[b] == K.OK:
                    assert length2[b] == length[b] + new[b] <= held[b] * bs
                    for i, s in enumerate(slots[cu[b]:cu[b] + new[b]]):
                        assert s == table[b][(length[b] + i) // bs] * bs + (length[b] + i) % bs
                else:
                    assert length2[b] == length[b] and all(s == -1 for s in slots[cu[b]:cu[b + 1]])
            length = length2
            done = [rng.random() < 0.1 for _ in range(B)]
            before = list(length)
            length, held, released, count, status = K.release(length, held, released, done, table, free, count, bs, window, sinks)
            assert status == [K.OK] * B
            live = []
            for b in range(B):
                mine = [j for j in range(held[b]) if not (j < released[b] and j * bs >= sinks)]
                live += [table[b][j] for j in mine]
                seen = {t // bs for t in range(length[b]) if window == 0 or length[b] - t < window or t < sinks}
                assert seen <= set(mine) and (not done[b] or before[b] == 0 or length[b] == 0)
            assert sorted(live + free[:count]) == list(range(nb))


def test_hand_worked():
    table = [[7, -1, -1], [-1, -1, -1], [-1, -1, -1]]
    r = K.extend([3, 0, 0], [3, 9, 1], [1, 0, 0], table, [5, 4, 3], 3, 4, 8, 20)
    # the first takes block 3, the second lacks one of three, the third comes behind it and gets none either
    assert r == ([0, 3, 12, 13], [31, 12, 13] + [-1] * 17, [6, 0, 0], [2, 0, 0], 2, [K.OK, K.ECAP, K.ECAP])
    assert table[0] == [7, 3, -1]
    # rows for the first only; the second keeps what it has, the third asks for nothing
    assert K.extend([3, 4, 5], [4, 9, 0], [1, 1, 1], [[1, 0], [2, 0], [3, 0]], [], 0, 8, 6, 6) == (
        [0, 4, 6, 6], [11, 12, 13, 14, -1, -1], [7, 4, 5], [1, 1, 1], 0, [K.OK, K.ECAP, K.OK])
    free = [9, -1, -1, -1, -1]
    r = K.release([40, 8], [5, 2], [0, 0], [False, True], [[1, 2, 3, 4, 5], [6, 7, 0, 0, 0]], free, 1, 8, 10, 3)
    # position 40 sees 31 ..: blocks 1 and 2 (tokens 8 .. 23) are behind it, block 0 holds the sinks
    assert r == ([40, 0], [5, 0], [3, 0], 5, [K.OK, K.OK]) and free == [9, 2, 3, 6, 7]
