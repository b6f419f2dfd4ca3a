"""A cache in pages, in plain terms (test oracle; see package header).

The paper takes the cache as given (Sec. 2.1). Here sequences may share a pool of pages [n_pages][n_kv][page][128]: row r of
a sequence is slot r % page of page table[r // page]; an entry outside [0, n_pages) is no page, and its rows are not there.
"""
import numpy as np


def places(table, n_pages, page, rows):
    """(page, slot) of each of the sequence's rows, page -1 where there is none."""
    out = []
    for r in rows:
        p = int(table[r // page]) if 0 <= r < len(table) * page else -1
        out.append((p if 0 <= p < n_pages else -1, r % page))
    return out


def rows_of(pool, table, kv_head, rows):
    """float64 rows of one KV head, zeroes where there is none, and which there are."""
    at = places(table, pool.shape[0], pool.shape[2], rows)
    there = np.array([p >= 0 for p, _ in at], bool)
    x = np.zeros((len(at), pool.shape[3]))
    for i, (p, slot) in enumerate(at):
        if p >= 0:
            x[i] = pool[p, kv_head, slot]
    return x, there


def sets(n, indexed, sink, window, ids):
    """Rows of the static set of a sequence of n tokens whose first `indexed` an index was built over, and the retrieved rows:
    entries of ids that are rows outside it, as often as they are given."""
    late = min(n - window, indexed)
    W = [r for r in range(n) if r < sink or r >= late]
    return np.array(W, np.int64), np.array([i for i in ids if 0 <= i < n and i not in set(W)], np.int64)
