"""Decode attention with sinks that are switched off, far away, or all that a request has:
against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from tests import attention_util as U
from tests import gpu_util as G
from tests.attention_edges import INF, LOWEST, SHAPES, agree, cache_of, decode, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,Hq,Hkv,D,shared,fp8", SHAPES)
def test_sinks_that_are_switched_off(lens, Hq, Hkv, D, shared, fp8):
    G.say(f"case: sinks of -inf and of the lowest value, lens={lens[:5]} heads {Hq}/{Hkv} D={D} shared={shared}")
    cache, q = cache_of(lens, Hkv, D, shared, fp8), U.queries(len(lens), Hq, D)
    for value in (-INF, LOWEST):
        sinks = torch.randn(Hq, device="cuda")
        sinks[::2] = value
        got, want = decode(cache, q, shared, sinks), reference(cache, q, shared, sinks)
        agree(got, want, cache, q, want[2])
        empty = np.array(lens) == 0
        assert not got[0][empty].any() and not np.isnan(got[0]).any()
        # a request with no visible slot has the sink's value
        assert np.array_equal(got[1][empty], np.broadcast_to(sinks.double().cpu().numpy(), (empty.sum(), Hq)))
        # a sink that is switched off is no sink
        none = decode(cache, q, shared)
        assert np.array_equal(got[0][~empty, ::2], none[0][~empty, ::2])


@pytest.mark.parametrize("lens", [[64, 40], [9000, 64]])
def test_sinks_of_requests_whose_pages_are_absent(lens):
    G.say(f"case: sinks of requests whose pages are all absent, lens={lens}")
    cache, q = cache_of(lens, 2, 128, (), False), U.queries(2, 8, 128)
    cache.table_np[0] = -1
    cache.table.copy_(torch.from_numpy(cache.table_np))
    sinks = torch.tensor([-INF, 3.0, LOWEST, -2.5] * 2, device="cuda")
    got, want = decode(cache, q, (), sinks), reference(cache, q, (), sinks)
    agree(got, want, cache, q, want[2])
    assert not got[0][0].any() and np.array_equal(got[1][0], sinks.double().cpu().numpy())


def test_sinks_far_above_and_below_the_scores():
    G.say("case: sinks of 1e30 and -1e30")
    lens = [0, 50, 3000]
    cache, q = cache_of(lens, 2, 64, (), False), U.queries(3, 4, 64)
    sinks = torch.tensor([1e30, -1e30, 500.0, 3e38], device="cuda")
    got, want = decode(cache, q, (), sinks), reference(cache, q, (), sinks)
    agree(got, want, cache, q, want[2])
    assert not got[0][:, [0, 3]].any()
