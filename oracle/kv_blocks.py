"""CPU oracle: block tables, slot maps and the list of free blocks, one sequence after the other.  TEST INFRASTRUCTURE ONLY."""
from __future__ import annotations

OK, EINVAL, ECAP = 0, -1, -3


def extend(length, new, held, table, free, count, block_size, num_blocks, cap):
    """All lists (table: a list of rows, changed in place).  Returns cu, slots, new length, new held, new count, status."""
    count = min(max(count, 0), len(free))
    cu, slots, new_length, new_held, status = [0], [-1] * cap, list(length), list(held), []
    rows, short = 0, False
    for b in range(len(length)):
        n, width = max(new[b], 0), len(table[b])
        first, rows = rows, rows + n
        cu.append(min(rows, cap))
        if length[b] < 0 or new[b] < 0 or held[b] < 0 or held[b] > width or length[b] > held[b] * block_size:
            status.append(EINVAL)
            continue
        want = max(0, -(-(length[b] + n) // block_size) - held[b])
        if length[b] + n > width * block_size or (n and rows > cap):
            status.append(ECAP)
            continue
        if want and (short or want > count):
            short = True
            status.append(ECAP)
            continue
        for j in range(want):
            count -= 1
            table[b][held[b] + j] = free[count]
        for i in range(n):
            pos = length[b] + i
            block = table[b][pos // block_size]
            slots[first + i] = block * block_size + pos % block_size if 0 <= block < num_blocks else -1
        new_length[b], new_held[b] = length[b] + n, held[b] + want
        status.append(OK)
    return cu, slots, new_length, new_held, count, status


def release(length, held, released, finished, table, free, count, block_size, window, sinks):
    """Changes ``free`` in place.  Returns new length, new held, new released, new count, status."""
    count = min(max(count, 0), len(free))
    new_length, new_held, new_released, status = list(length), list(held), list(released), []
    full = False
    for b in range(len(length)):
        if not (0 <= held[b] <= len(table[b]) and 0 <= length[b] <= held[b] * block_size and 0 <= released[b] <= held[b]):
            status.append(EINVAL)
            continue

        def gone(j):            # given back before
            return j < released[b] and j * block_size >= sinks

        def unseen(j):          # no token of block j is a sink or within the window of position length[b]
            return all(t >= sinks and length[b] - t >= window for t in (j * block_size, (j + 1) * block_size - 1))
        if finished[b]:
            give = [j for j in range(held[b]) if not gone(j)]
        else:
            give = [j for j in range(held[b]) if window > 0 and not gone(j) and unseen(j)]
        if give and (full or len(give) > len(free) - count):
            full = True
            status.append(ECAP)
            continue
        for j in give:
            free[count] = table[b][j]
            count += 1
        if finished[b]:
            new_length[b] = new_held[b] = new_released[b] = 0
        elif give:
            new_released[b] = give[-1] + 1
        status.append(OK)
    return new_length, new_held, new_released, count, status
