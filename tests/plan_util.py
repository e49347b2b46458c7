"""The books of a paged cache, kept one sequence after the other on the host."""
import numpy as np

from tree_util import as_words, branch


def plan(new, lengths, table, free, count, page, rows, parents=None, words=1):
    """Lists and a table as numpy; returns (starts, totals, slots, positions, masks or None, table, free, count)."""
    table, free, pages = np.array(table), list(free), len(free)
    width = table.shape[1]
    left = min(max(count, 0), pages)
    for s, n in enumerate(new):
        if n < 0:
            for p in table[s]:
                if 0 <= p < pages and left < pages:
                    free[left] = int(p)
                    left += 1
            table[s] = -1
    starts, totals, slots, positions, masks = [0], [], [], [], []
    for s, (n, length) in enumerate(zip(new, lengths)):
        base = 0 if n < 0 else min(max(length, 0), 1 << 30)
        n = max(n, 0)
        lack = []
        fits = n <= rows - starts[-1] and base + n <= width * page
        if n and fits:
            lack = [c for c in range(base // page, (base + n - 1) // page + 1) if not 0 <= table[s, c] < pages]
            fits = len(lack) <= left
        if not fits:
            n, lack = 0, []
        for c in lack:
            left -= 1
            table[s, c] = free[left]
        up = []
        for t in range(n):
            u = int(parents[s][t]) if parents is not None and t < len(parents[s]) else -1
            up.append(u if 0 <= u < t else -1)
        for t in range(n):
            p = int(table[s, (base + t) // page])
            slots.append(p * page + (base + t) % page if 0 <= p < pages else -1)
            tree = parents is not None and n <= 64 * words
            path = branch(up, t) if tree else []
            positions.append(base + len(path) - 1 if tree else base + t)
            masks.append(sum(1 << j for j in path))
        starts.append(starts[-1] + n)
        totals.append(base + n)
    behind = rows - starts[-1]
    slots, positions, masks = slots + [-1] * behind, positions + [-1] * behind, masks + [0] * behind
    return starts, totals, slots, positions, as_words(masks, words) if parents is not None else None, table, free, left
