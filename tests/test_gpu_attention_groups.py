"""Groups that share a prefix: where the first members are empty, and where pages inside
the prefix are absent."""
import numpy as np
import pytest
import torch

from oracle import attention as A
from paper_2607_00466_amd import binding as B
from tests import attention_util as U
from tests import gpu_util as G

pytestmark = pytest.mark.gpu


def _check_weights(cache, q, lse, shared):
    R, Hq, D = q.shape
    gs, pl, gs_np, pl_np = U.groups_of(shared, R)
    w_in, out = torch.rand((R, cache.Hkv, cache.N), device="cuda"), torch.full((R, cache.Hkv, cache.N), -2.0, device="cuda")
    before = out.double().cpu().numpy()
    want = A.weights(q.double().cpu().numpy(), cache.k_np, cache.table_np, cache.lens_np, lse.double().cpu().numpy(), D ** -0.5,
                     w_in.double().cpu().numpy(), before, gs_np, pl_np)
    B.moe_attn_weights(q, cache.k, cache.table, cache.lens, lse, cache.dims(Hq), w_in, out, gs, pl, cache.k_scale)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    # as test_weights: the exponent's error over the heads' weights, and the additions' roundings
    tol = (np.expm1(U.score_bound(q, cache, D ** -0.5)) + (Hq // cache.Hkv + 64) * U.U_FP32) * (np.abs(want) + 1)
    assert (np.abs(got - want) <= tol).all()


# lens; the group; its first member that holds anything
EMPTY_FIRST = [
    ([0, 80, 64, 70], (0, 4, 64), 1, 8, 1, 128, False),
    ([0, 0, 0, 300, 290, 0, 257], (0, 7, 256), 3, 32, 4, 128, False),
    ([40, 0, 300, 257, 0, 700], (1, 6, 250), 2, 8, 2, 64, True),
    ([0, 533, 530], (0, 3, 512), 1, 16, 2, 256, True),
    ([0, 150, 140], (0, 3, 128), 1, 24, 1, 128, False),    # more than 16 heads a kv head
    ([50, 0, 0, 20], (1, 3, 48), 1, 8, 2, 64, False),      # a group of empty requests
    ([0, 90], (0, 2, 64), 1, 3, 3, 64, False),
]


@pytest.mark.parametrize("lens,group,holder,Hq,Hkv,D,fp8", EMPTY_FIRST)
@pytest.mark.parametrize("stale", [False, True])
def test_a_prefix_is_read_through_the_first_member_that_holds_it(lens, group, holder, Hq, Hkv, D, fp8, stale):
    G.say(f"case: a group whose first members are empty, lens={lens} group={group} heads {Hq}/{Hkv} D={D} stale={stale}")
    s, e, tokens = group
    cache = U.Cache(lens, Hkv, D, 16, fp8, seed=D, shared=((holder, e, tokens),), max_blocks=-(-max(lens) // 16) + 1)
    if stale:
        # an empty request's row still names pages: other requests' and unused ones
        rng = np.random.default_rng(1)
        for r, n in enumerate(lens):
            if n == 0:
                cache.table_np[r] = rng.integers(0, cache.nb, cache.max_blocks)
        cache.table.copy_(torch.from_numpy(cache.table_np))
    q = U.queries(len(lens), Hq, D)
    _, lse = U.run_decode(cache, q, (group,))
    _check_weights(cache, q, lse, (group,))


@pytest.mark.parametrize("D,fp8,bs", [(128, False, 16), (64, True, 32), (256, False, 16)])
def test_absent_pages_inside_a_prefix(D, fp8, bs):
    G.say(f"case: holes in a shared prefix on both sides of slot 1024, D={D} fp8={fp8} bs={bs}")
    lens, group = [2300, 2200, 2250, 2177], (0, 4, 2176)
    cache = U.Cache(lens, 2, D, bs, fp8, seed=D, shared=(group,), max_blocks=2304 // bs)
    # single pages, a whole 64-slot stage, pages on both sides of slot 1024, a run over slots 1920 to 2111
    for lo, hi in ((0, 16), (80, 96), (320, 384), (1008, 1040), (1920, 2112)):
        cache.table_np[0, lo // bs:-(-hi // bs)] = -1
    cache.table_np[0, 700 // bs] = cache.nb + 3
    cache.table.copy_(torch.from_numpy(cache.table_np))
    q = U.queries(4, 16, D)
    _, lse = U.run_decode(cache, q, (group,))
    _check_weights(cache, q, lse, (group,))
