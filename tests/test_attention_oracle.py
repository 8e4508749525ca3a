"""The attention oracle against closed forms, brute force and its own invariants (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import attention as A


def _cache(rng, nb, Hkv, bs, D):
    return rng.standard_normal((nb, Hkv, bs, D))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_product_of_complex_numbers(interleaved):
    rng = np.random.default_rng(0)
    T, H, D, half = 5, 2, 24, 8
    x = rng.standard_normal((T, H, D))
    pos = rng.integers(0, 50, (2, T))
    axis = np.array([0, 1] * 4)
    angle = np.arange(50)[:, None] * 0.3 ** np.arange(half)
    y = A.rotate(x, pos, axis, np.cos(angle), np.sin(angle), interleaved)
    lo = 2 * np.arange(half) if interleaved else np.arange(half)
    hi = lo + 1 if interleaved else lo + half
    for t in range(T):
        turn = np.exp(1j * pos[axis, t] * 0.3 ** np.arange(half))
        assert np.allclose(y[t, :, lo].T + 1j * y[t, :, hi].T, (x[t, :, lo].T + 1j * x[t, :, hi].T) * turn)
    assert np.array_equal(y[..., 16:], x[..., 16:])
    assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1))


def test_scores_of_rotated_rows_depend_on_the_distance_alone():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 16))
    angle = np.arange(100)[:, None] * 0.5 ** np.arange(8)
    dot = [float((A.rotate(q, [[p + 7]], [0] * 8, np.cos(angle), np.sin(angle)) *
                  A.rotate(k, [[p]], [0] * 8, np.cos(angle), np.sin(angle))).sum()) for p in (0, 13, 88)]
    assert np.allclose(dot, dot[0])


def test_positions_outside_the_table_are_nan():
    x = np.ones((2, 1, 16))
    y = A.rotate(x, [[5, -1]], [0] * 7 + [3], np.ones((6, 8)), np.zeros((6, 8)))
    assert np.isnan(y[1]).all()
    assert np.isnan(y[0, 0, [7, 15]]).all() and not np.isnan(y[0, 0, :7]).any()


def test_decode_against_a_dense_softmax():
    rng = np.random.default_rng(2)
    R, Hq, Hkv, D, bs, nb = 3, 6, 2, 8, 4, 20
    k, v, q = _cache(rng, nb, Hkv, bs, D), _cache(rng, nb, Hkv, bs, D), rng.standard_normal((R, Hq, D))
    table = rng.permutation(nb)[:R * 5].reshape(R, 5)
    lens = [20, 7, 0]
    sinks = rng.standard_normal(Hq)
    for window, sink in ((0, None), (0, sinks), (5, None)):
        out, lse, _ = A.decode(q, k, v, table, lens, 0.3, sinks=sink, window=window)
        for r in range(2):
            K, V = (c[table[r]].transpose(1, 0, 2, 3).reshape(Hkv, 20, D) for c in (k, v))
            s = torch.tensor(np.einsum("hgd,hjd->hgj", q[r].reshape(Hkv, 3, D), K) * 0.3)
            j = torch.arange(20)
            s[..., (j >= lens[r]) | ((j < lens[r] - window) if window else (j < 0))] = -math.inf
            if sink is not None:
                s = torch.cat([s, torch.tensor(sink).view(Hkv, 3, 1)], -1)
            p = s.softmax(-1)[..., :20]
            assert np.allclose(out[r].reshape(Hkv, 3, D), p.numpy() @ V)
            assert np.allclose(lse[r].reshape(Hkv, 3), s.logsumexp(-1))
        assert not out[2].any() and np.array_equal(lse[2], np.full(Hq, -np.inf) if sink is None else sink)


def test_equal_keys_average_the_values_and_absent_pages_do_not_count():
    rng = np.random.default_rng(3)
    k, v = np.ones((4, 1, 4, 8)), _cache(rng, 4, 1, 4, 8)
    out, lse, mass = A.decode(np.ones((1, 1, 8)), k, v, [[2, -1, 0, 9]], [16], 1.0)
    rows = np.concatenate([v[2, 0], v[0, 0]])
    assert np.allclose(out[0, 0], rows.mean(0)) and np.allclose(lse, 8 + math.log(8))
    assert np.allclose(mass[0, 0], np.abs(rows).mean(0))


def test_a_shared_prefix_is_read_through_the_first_member():
    rng = np.random.default_rng(4)
    k, v, q = _cache(rng, 9, 1, 4, 8), _cache(rng, 9, 1, 4, 8), rng.standard_normal((3, 1, 8))
    # members 1 and 2 hold nothing of their own in the first page
    shared = A.decode(q, k, v, [[0, 1], [-1, 2], [-1, 3]], [6, 8, 7], 1.0, [0, 3], [4])
    own = A.decode(q, k, v, [[0, 1], [0, 2], [0, 3]], [6, 8, 7], 1.0)
    assert all(np.array_equal(a, b) for a, b in zip(shared, own))
    # shared as far as the shortest member that holds anything
    assert A.shared_reach([6, 0, 3], [0, 3], [4], 8) == [(0, 3)] * 3
    assert A.shared_reach([6, 5], [0, 1, 2], [4, 4], 8) == [(0, 0), (1, 0)]
    assert A.shared_reach([6, 5, 9, 9], [1, 3, 9], [4, 5], 8) == [(0, 0), (1, 4), (1, 4), (3, 0)]


def test_weights_of_a_request_sum_to_its_heads():
    rng = np.random.default_rng(5)
    k, q = _cache(rng, 6, 2, 4, 8), rng.standard_normal((2, 4, 8))
    table = [[0, 1, 2], [3, 4, 5]]
    _, lse, _ = A.decode(q, k, k, table, [12, 5], 0.7)
    w0 = rng.random((2, 2, 12))
    w = A.weights(q, k, table, [12, 5], lse, 0.7, w0, w0)
    assert np.allclose((w - w0).sum(-1), 2.0)
    assert np.array_equal(w[1, :, 5:], w0[1, :, 5:])


def test_evict_keeps_the_heaviest_and_fills_the_holes_in_order():
    w = np.array([[[5, 0, 9, 1, 0, 7, 2, 0.]]])
    pos = np.arange(8)[None, None]
    src, new, w2, p2 = A.evict(w, pos, [8], [8], 4, 1)
    # slot 7 is recent; 2, 5 and 0 are the heaviest
    assert src[0, 0].tolist() == [0, 5, 2, 7] and new.tolist() == [4]
    assert w2[0, 0].tolist() == [5, 7, 9, 0, 0, 0, 0, 0] and p2[0, 0].tolist() == [0, 5, 2, 7, -1, -1, -1, -1]
    # equal weights: the lowest slots stay, nothing moves
    src, *_ = A.evict(np.zeros((1, 1, 8)), pos, [8], [100], 4, 0)
    assert src[0, 0].tolist() == [0, 1, 2, 3]
    # under the budget nothing changes
    src, new, w2, p2 = A.evict(w, pos, [3], [8], 4, 1)
    assert src[0, 0].tolist() == [0, 1, 2, -1] and np.array_equal(w2, w) and new.tolist() == [3]


def test_moved_rows_follow_src():
    rng = np.random.default_rng(6)
    cache = _cache(rng, 5, 2, 4, 3)
    table = [[4, 1, 0]]
    src = np.array([[[0, 9, 2, 3, 8], [0, 1, 2, 3, 4]]])
    after = A.moved(cache, table, src, [10], 5)
    want = cache.copy()
    want[4, 0, 1], want[1, 0, 0] = cache[0, 0, 1], cache[0, 0, 0]
    assert np.array_equal(after, want)
