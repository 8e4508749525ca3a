"""Accumulated weights may start at any element of their allocation."""
import pytest
import torch

from paper_2607_00466_amd import binding as B
from tests import attention_util as U
from tests import gpu_util as G

pytestmark = pytest.mark.gpu


def test_weights_and_evict_take_arrays_at_any_element():
    G.say("case: accumulated weights that start at an odd element of their allocation")
    cache = U.Cache([100, 40], 2, 64, 16, seed=3)
    q = U.queries(2, 4, 64)
    d = cache.dims(4)
    _, lse = U.run_decode(cache, q)
    shape, n = (2, 2, cache.N), 4 * cache.N

    def weights(skip):
        """weights_in, weights_out and evict's weights_out, `skip` elements into their memory."""
        g = torch.Generator(device="cuda").manual_seed(1)
        given = torch.rand(n, device="cuda", generator=g)
        return [torch.cat([torch.zeros(skip, device="cuda"), x])[skip:].view(shape) for x in (given, given * 0, given * 0)]

    got = []
    for skip in (0, 1):
        w_in, w_out, w_kept = weights(skip)
        B.moe_attn_weights(q, cache.k, cache.table, cache.lens, lse, d, w_in, w_out)
        pos = torch.arange(cache.N, device="cuda", dtype=torch.int32).expand(shape).contiguous()
        src, new = torch.empty((2, 2, 30), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
        B.moe_kv_evict(w_out, pos, cache.lens, cache.lens, cache.table, d, 30, 3, cache.k.clone(), cache.v.clone(), src, new,
                       w_kept, pos)
        got.append((w_out, w_kept, src, new, pos))
    assert got[0][0].data_ptr() % 16 == 0 and got[1][0].data_ptr() % 16 == 4
    assert all(torch.equal(a, b) for a, b in zip(*got))
