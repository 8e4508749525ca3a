"""Eviction from tables far wider than the requests' caches: what is done for a row is
decided by its length, whatever the table could hold."""
import numpy as np
import pytest
import torch

from oracle import attention as A
from paper_2607_00466_amd import binding as B
from tests import attention_util as U
from tests import gpu_util as G

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,budget,max_blocks", [
    # a few tokens over the budget, many, none, in tables of each selection's size
    ([101, 164, 165, 500, 100, 0], 100, 32),
    ([1025, 1088, 1089, 2000, 1024, 3], 1024, 128),
    ([300, 900, 268, 269], 205, 512),
    ([2049, 6000, 2000], 2048, 2048),
    # tables past 32,768 slots: short rows, few moves, long rows
    ([1025, 1089, 5000, 1024, 0], 1024, 4096),
    ([33000, 32768, 32769, 40, 36000], 32736, 4096),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_from_wide_tables(lens, budget, max_blocks, in_place):
    G.say(f"case: evict lens={lens} budget={budget} from tables of {max_blocks} pages, in_place={in_place}")
    R, Hkv, recent, gap = len(lens), 2, 7, 40
    cache = U.Cache(lens, Hkv, 64, 16, seed=budget, max_blocks=max_blocks)
    rng = np.random.default_rng(budget)
    N = cache.N
    w = np.floor(rng.exponential(1.0, (R, Hkv, N)) * 3).astype(np.float32)  # many equal ones
    pos = np.broadcast_to(np.arange(N, dtype=np.int32) + gap * (rng.random((R, Hkv, N)) < 0.5), w.shape).astype(np.int32)
    seen = np.array([n + gap for n in lens], np.int32)
    protect = np.array([3 * r for r in range(R)], np.int32)
    src, new, w2, p2 = A.evict(w, pos, lens, seen, budget, recent, protect)
    want = [A.moved(c.float().cpu().numpy(), cache.table_np, src, lens, budget) for c in (cache.k, cache.v)]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    w_d, p_d = dev(w), dev(pos)
    w_out, p_out = (w_d, p_d) if in_place else (dev(w), dev(pos))
    src_d = torch.full((R, Hkv, budget), -9, dtype=torch.int32, device="cuda")
    new_d = torch.empty(R, dtype=torch.int32, device="cuda")
    B.moe_kv_evict(w_d, p_d, cache.lens, dev(seen), cache.table, cache.dims(Hkv), budget, recent, cache.k, cache.v, src_d, new_d,
                   w_out, p_out, protect=dev(protect))
    torch.cuda.synchronize()
    assert np.array_equal(src_d.cpu().numpy(), src)
    assert np.array_equal(new_d.cpu().numpy(), new)
    assert np.array_equal(w_out.cpu().numpy(), w2)
    assert np.array_equal(p_out.cpu().numpy(), p2)
    for got, ref in zip((cache.k, cache.v), want):
        assert np.array_equal(got.float().cpu().numpy(), ref, equal_nan=True)
