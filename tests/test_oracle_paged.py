"""Hand-worked cases of the oracle of a cache in pages."""
import numpy as np

from oracle import paged as OP


def test_rows_by_hand():
    pool = np.arange(4 * 1 * 2 * 1, dtype=np.float64).reshape(4, 1, 2, 1)          # page p holds 2 p and 2 p + 1
    x, there = OP.rows_of(pool, [3, -1, 0, 4], 0, [0, 1, 2, 4, 5, 6, 8, -1])
    assert there.tolist() == [True, True, False, True, True, False, False, False]
    assert x[:, 0].tolist() == [6, 7, 0, 0, 1, 0, 0, 0]


def test_sets_by_hand():
    W, om = OP.sets(10, 7, 2, 2, [5, 1, 6, 7, 9, -1, 10, 5, 2])
    assert W.tolist() == [0, 1, 7, 8, 9] and om.tolist() == [5, 6, 5, 2]
    assert OP.sets(10, 10, 2, 3, [])[0].tolist() == [0, 1, 7, 8, 9]
    assert OP.sets(4, 4, 3, 3, [1])[0].tolist() == [0, 1, 2, 3] and OP.sets(4, 4, 3, 3, [1])[1].size == 0
    assert OP.sets(0, 0, 3, 3, [0])[0].size == 0
