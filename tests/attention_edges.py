"""Shapes and comparisons of the attention tests whose inputs or outputs need not be finite."""
from __future__ import annotations

import numpy as np

from oracle import attention as A
from tests import attention_util as U

INF, NAN, LOWEST = float("inf"), float("nan"), float(np.finfo(np.float32).min)

# lens, Hq, Hkv, D, shared, fp8: one segment a request and many, empty requests, a
# group with an empty member, and every join (9000 slots of few rows, 1050 rows)
SHAPES = [
    ([0, 1, 40, 300], 8, 2, 128, (), False),
    ([0, 9000], 4, 4, 64, (), False),
    ([700, 0, 33], 16, 2, 256, (), True),
    ([5, 0] * 75, 7, 1, 64, (), True),
    ([200, 0, 170, 150], 32, 4, 128, ((0, 4, 128),), False),
    ([600, 590, 0], 8, 1, 64, ((0, 3, 576),), True),
]


def cache_of(lens, Hkv, D, shared, fp8):
    return U.Cache(lens, Hkv, D, 16, fp8, seed=len(lens) + D, shared=shared, max_blocks=-(-max(lens) // 16) + 1)


def decode(cache, q, shared, sinks=None):
    out, lse = U.run_decode(cache, q, shared, sinks, check=False)
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def reference(cache, q, shared, sinks=None):
    _, _, gs, pl = U.groups_of(shared, q.shape[0])
    with np.errstate(invalid="ignore"):
        return A.decode(q.double().cpu().numpy(), cache.k_np, cache.v_np, cache.table_np, cache.lens_np, cache.D ** -0.5, gs, pl,
                        None if sinks is None else sinks.double().cpu().numpy())


def _same_places(got, want):
    """NaN and each infinity where the reference has them; the places that are finite."""
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got == INF, want == INF) and np.array_equal(got == -INF, want == -INF)
    return np.isfinite(want)


def agree(got, want, cache, clean_q, mass):
    """As check_decode, where the reference is finite; mass and the queries of the inputs
    without what was planted bound the errors of the rest."""
    e = U.score_bound(clean_q, cache, cache.D ** -0.5)
    ok = _same_places(got[1], want[1])
    assert (np.abs(got[1] - want[1])[ok] <= (e + 16 * U.U_FP32 * (1 + np.abs(want[1])))[ok]).all()
    ok = _same_places(got[0], want[0])
    tol = (U.U_BF16 + np.expm1(2 * e) + 64 * U.U_FP32) * mass * 1.01 + U.U_BF16 * 1.01 * np.abs(want[0]) + 1e-38
    assert (np.abs(got[0] - want[0])[ok] <= tol[ok]).all()
