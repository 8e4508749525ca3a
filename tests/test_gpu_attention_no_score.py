"""Decode attention of requests whose every score is -inf: as without a visible slot."""
import pytest
import torch

from tests import attention_util as U
from tests import gpu_util as G
from tests.attention_edges import INF, cache_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,Hq,Hkv,D,shared", [([40, 9000, 0], 8, 2, 128, ()), ([300, 290], 4, 1, 64, ((0, 2, 256),))])
def test_scores_of_minus_infinity_alone(lens, Hq, Hkv, D, shared):
    G.say(f"case: every score -inf, lens={lens} heads {Hq}/{Hkv} D={D} shared={shared}")
    cache, q = cache_of(lens, Hkv, D, shared, False), U.queries(len(lens), Hq, D)
    cache.k[..., 5] = -INF  # (slots that do not count hold anything)
    q[..., 5] = q[..., 5].abs() + 1
    sinks = torch.linspace(-3, 4, Hq, device="cuda")
    for s, value in ((None, torch.full((Hq,), -INF, device="cuda")), (sinks, sinks)):
        out, lse = U.run_decode(cache, q, shared, s, check=False)
        assert not out.any() and torch.equal(lse, value.expand_as(lse))
