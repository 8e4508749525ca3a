"""The attention oracle where groups have empty members and sums are empty (CPU)."""
import numpy as np

from oracle import attention as A


def test_a_prefix_is_read_through_the_first_member_that_holds_anything():
    assert A.shared_reach([0, 6, 3], [0, 3], [4], 8) == [(1, 3)] * 3
    assert A.shared_reach([5, 0, 0, 7, 9], [1, 5], [4], 8) == [(0, 0)] + [(3, 4)] * 4
    rng = np.random.default_rng(0)
    k, v, q = (rng.standard_normal(s) for s in ((5, 1, 4, 8), (5, 1, 4, 8), (3, 1, 8)))
    # the empty first member's row names a page of something else
    shared = A.decode(q, k, v, [[4, 4], [0, 1], [-1, 2]], [0, 6, 7], 1.0, [0, 3], [4])
    own = A.decode(q, k, v, [[4, 4], [0, 1], [0, 2]], [0, 6, 7], 1.0)
    assert all(np.array_equal(a, b) for a, b in zip(shared, own))


def test_a_sink_that_is_switched_off_is_none():
    rng = np.random.default_rng(1)
    k, v, q = (rng.standard_normal(s) for s in ((2, 1, 4, 8), (2, 1, 4, 8), (2, 2, 8)))
    table, lens = [[0], [1]], [3, 0]
    none = A.decode(q, k, v, table, lens, 1.0)
    off = A.decode(q, k, v, table, lens, 1.0, sinks=[-np.inf, -np.inf])
    assert all(np.array_equal(a, b) for a, b in zip(none, off))
    assert np.array_equal(off[1][1], [-np.inf] * 2) and not off[0][1].any()
