"""The oracle of the int8 cache, forks and compaction against closed forms (no GPU)."""
import numpy as np
import pytest

from oracle import kv_cache as K


def test_norm_is_the_unit_mean_square():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 3, 64)).astype(np.float32)
    y = K.normed(x, np.ones(64), 0.0, exact=True)
    np.testing.assert_allclose((y * y).mean(-1), 1.0, rtol=1e-12)
    # without eps it does not depend on the row's size; powers of two change no bit
    np.testing.assert_array_equal(K.normed(x * 8, np.ones(64), 0.0), K.normed(x, np.ones(64), 0.0))
    assert K.normed(x, None, 1.0) is not None and np.array_equal(K.normed(x, None, 1.0), x)
    np.testing.assert_allclose(K.normed(np.full((1, 4), 3.0), np.arange(4), 16.0, exact=True), [3 / 5 * np.arange(4)], rtol=1e-12)


def test_turn_by_a_quarter():
    x = np.arange(8, dtype=np.float32).reshape(1, 1, 8)
    cos, sin = np.zeros((1, 2)), np.ones((1, 2))
    y = K.turned(x, [[0]], [0, 0], cos, sin)
    np.testing.assert_array_equal(y[0, 0], [-2, -3, 0, 1, 4, 5, 6, 7])
    y = K.turned(x, [[0]], [0, 0], cos, sin, interleaved=True)
    np.testing.assert_array_equal(y[0, 0], [-1, 0, -3, 2, 4, 5, 6, 7])


def _empty(nb=3, Hkv=1, bs=16, D=4):
    return np.zeros((nb, Hkv, bs, D), np.int8), np.zeros((nb, Hkv), np.float32)


def test_a_fresh_page_uses_all_of_its_codes():
    codes, scale = _empty()
    x = np.array([[[1.0, -2.0, 0.5, 0.0]]], np.float32)
    codes, scale = K.append_int8(x, [0, 1], [[2]], [0], codes, scale)
    assert scale[2, 0] == np.float32(2) * (np.float32(1) / np.float32(127))
    assert codes[2, 0, 0].tolist() == [64, -127, 32, 0]  # 63.5 and 31.75


def test_growth_by_powers_of_two_and_a_step_at_most():
    rng = np.random.default_rng(1)
    codes, scale = _empty(D=64)
    rows = rng.standard_normal((16, 1, 64)).astype(np.float32) * (1.6 ** np.arange(16, dtype=np.float32))[:, None, None]
    scales = []
    for j in range(16):
        codes, scale = K.append_int8(rows[j:j + 1], [0, 1], [[0]], [j], codes, scale)
        scales.append(float(scale[0, 0]))
        # never more than a step off, and half of one where it has just been written
        off = np.abs(codes[0, 0, :j + 1] * np.float64(scale[0, 0]) - rows[:j + 1, 0])
        assert off.max() <= scale[0, 0] and off[j].max() <= scale[0, 0] * (0.5 + 1e-5)
    grew = np.log2(np.array(scales) / scales[0])
    assert np.array_equal(grew, np.rint(grew)) and grew[-1] >= 7 and (np.diff(grew) >= 0).all()


def test_pages_and_rows_that_receive_nothing():
    rng = np.random.default_rng(2)
    codes, scale = rng.integers(-128, 128, (4, 2, 16, 4)).astype(np.int8), rng.random((4, 2)).astype(np.float32)
    x = rng.standard_normal((40, 2, 4)).astype(np.float32)
    after, s = K.append_int8(x, [0, 20, 20, 40], [[0, 1], [2, 2], [9, 3]], [15, 3, 14], codes, scale)
    np.testing.assert_array_equal(after[2], codes[2])             # a request without tokens
    # (the third request's first two tokens fall into page 9, which is absent)
    assert (s[2] == scale[2]).all() and s[3, 0] == np.abs(x[22:38, 0]).max() * (np.float32(1) / np.float32(127))


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_what_is_not_finite_makes_the_page_nan(bad):
    codes, scale = _empty()
    x = np.ones((2, 1, 4), np.float32)
    x[1, 0, 2] = bad
    codes, scale = K.append_int8(x, [0, 2], [[0]], [0], codes, scale)
    assert np.isnan(scale[0, 0])
    codes, scale = K.append_int8(x[:1], [0, 1], [[0]], [2], codes, scale)  # and it stays so
    assert np.isnan(scale[0, 0])
    codes, scale = K.append_int8(x[:1], [0, 1], [[0]], [0], codes, scale)  # until it is begun anew
    assert scale[0, 0] == np.float32(1) / np.float32(127)


def test_fork_shares_full_pages():
    cache = np.arange(6 * 16, dtype=np.float32).reshape(1, 6, 1, 16, 1)
    table = np.array([[0, 1, 2], [-1, -1, -1], [5, 5, 5]], np.int32)
    t, n, (c,), _ = K.fork([0], [1], [4], table, np.array([35, 0, 7]), [cache])
    assert t.tolist() == [[0, 1, 2], [0, 1, 4], [5, 5, 5]] and n.tolist() == [35, 35, 7]
    np.testing.assert_array_equal(c[0, 4, 0, :3], cache[0, 2, 0, :3])
    np.testing.assert_array_equal(c[0, 4, 0, 3:], cache[0, 4, 0, 3:])
    t, n, (c,), _ = K.fork([0], [1], [4], table, np.array([32, 0, 7]), [cache])  # no page is partly filled
    assert t[1].tolist() == [0, 1, -1]
    np.testing.assert_array_equal(c, cache)


def test_compact_moves_into_free_pages_only():
    cache = np.arange(5, dtype=np.float32).reshape(1, 5, 1, 1, 1)
    table = np.array([[4, 3, 0, -1, 7]], np.int32)
    t, (c,), _ = K.compact([0, -1, 9, 3, 1], table, [cache])
    assert t.tolist() == [[1, 3, 0, -1, -1]] and c[0, :, 0, 0, 0].tolist() == [0, 4, 2, 3, 4]
    t, (c,), _ = K.compact([0, -1, -1, 0, 3], table, [cache])  # 0 and 3 are held: nothing moves there
    assert t.tolist() == [[4, 3, 0, -1, -1]] and c[0, :, 0, 0, 0].tolist() == [0, 1, 2, 3, 4]
