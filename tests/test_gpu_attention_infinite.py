"""Decode attention over infinite values in cached slots: against the 64-bit oracle."""
import pytest

from tests import attention_util as U
from tests import gpu_util as G
from tests.attention_edges import INF, agree, cache_of, decode, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,Hq,Hkv,D,shared", [
    ([9000], 4, 4, 64, ()), ([700, 33], 16, 2, 256, ()), ([17000, 5], 8, 1, 128, ()),
    ([900, 800, 810], 32, 4, 128, ((0, 3, 640),)),
    ([3000] * 70, 16, 1, 64, ()),
])
def test_visible_values_that_are_infinite(lens, Hq, Hkv, D, shared):
    # (scores near each other: no weight is too small for 32 bits, so an infinite value's column is infinite)
    G.say(f"case: infinite values in cached slots, lens={lens[:5]} heads {Hq}/{Hkv} D={D} shared={shared}")
    cache, q = cache_of(lens, Hkv, D, shared, False), U.queries(len(lens), Hq, D, amp=0.5)
    clean = reference(cache, q, shared)
    for r, n in enumerate(lens):
        for i, j in enumerate((n - 1, n // 2)):
            b = int(cache.table_np[r if not shared or j >= shared[0][2] else 0, j // 16])
            for c in (cache.v, cache.v_np):
                c[b, 0, j % 16, 7 + i] = -INF if (r + i) % 2 else INF
    agree(decode(cache, q, shared), reference(cache, q, shared), cache, q, clean[2])
