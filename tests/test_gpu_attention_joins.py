"""moe_attn_decode's joins: which kernel adds a row's parts up goes by how many rows there
are (1024, and 4096 where D is 128 or 256) and, where D is 64, by how many parts a
request's rows have.  Row counts around the limits, the last workgroup partly filled,
rows without a part, with one, with a few and with many, of their own and of a prefix."""
import numpy as np
import pytest
import torch

from paper_2607_00466_amd import binding as B
from tests import attention_util as U
from tests.test_gpu_attention_int8 import Cache as Int8Cache

pytestmark = pytest.mark.gpu

KINDS = {"bf16": lambda *a, **kw: U.Cache(*a, **kw), "fp8": lambda *a, **kw: U.Cache(*a, fp8=True, **kw), "int8": Int8Cache}


def lengths(R, seed=0, top=60):
    """R requests: most of them short, some empty, a few of several parts and one of many."""
    rng = np.random.default_rng(seed)
    n = rng.integers(1, top, R)
    n[rng.random(R) < 0.15] = 0
    n[[1, R // 2, R - 1]] = 700, 500, 1100
    n[R // 3] = 3300
    return [int(x) for x in n]


def check(kind, lens, Hq, Hkv, D, shared=(), sinks=False, seed=0):
    c = KINDS[kind](lens, Hkv, D, 16, seed=seed, shared=shared)
    s = torch.randn(Hq, generator=torch.Generator().manual_seed(seed)).cuda() * 3 if sinks else None
    return c, U.run_decode(c, U.queries(len(lens), Hq, D, seed), shared, s)


# rows: 1022, 1024, 1029, 1040
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("R,Hq,Hkv", [(146, 7, 1), (64, 16, 2), (147, 7, 1), (65, 16, 4)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_around_1024_rows(kind, R, Hq, Hkv, D):
    check(kind, lengths(R, R), Hq, Hkv, D, sinks=D == 128, seed=R)


# rows: 4088, 4096, 4102, 4128
@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("R,Hq,Hkv", [(292, 14, 2), (128, 32, 4), (293, 14, 1), (129, 32, 2)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_around_4096_rows(kind, R, Hq, Hkv, D):
    check(kind, lengths(R, R + 1, 40), Hq, Hkv, D, sinks=D != 128, seed=R)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,R", [(64, 70), (128, 140), (256, 140)])
def test_parts_of_prefixes_and_of_their_own(kind, D, R):
    """More rows than either limit; a prefix in many parts for two members, another in few
    for many, a group of which a member is empty."""
    lens = lengths(R, 3)
    shared = [(0, 2, 2560), (4, 20, 320), (30, 34, 128)]
    lens[0], lens[1] = 2600, 4000
    for r in range(4, 20):
        lens[r] = 320 + 13 * (r - 4)
    lens[30:34] = 128, 200, 0, 700
    check(kind, lens, 32, 2, D, shared, sinks=True, seed=D)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens,Hq,Hkv", [
    ([3000] * 70, 16, 1),                # every row in many parts, more of them than waves
    ([20_000] + [3] * 33, 32, 1),        # one request alone
    ([2] * 40 + [0] * 5 + [9000], 64, 8),
    ([6000] * 3 + [1500] * 20 + [7] * 30, 20, 2),
])
def test_rows_of_many_parts_where_D_is_64(kind, lens, Hq, Hkv):
    check(kind, lens, Hq, Hkv, 64, seed=len(lens))


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("D", [128, 256])
def test_the_bits_of_a_row_are_those_of_either_join(kind, D):
    """4096 rows, and as many with an empty request behind them: the same parts, added in
    the same order by 64 threads a row and by D / 4."""
    lens = lengths(128, 5)
    c, (out, lse) = check(kind, lens, 32, 4, D)
    more = KINDS[kind](lens + [0], 4, D, 16, seed=0)
    more.k, more.v, more.k_scale, more.v_scale, more.nb = c.k, c.v, c.k_scale, c.v_scale, c.nb
    more.table = torch.cat([c.table, torch.full((1, c.max_blocks), -1, dtype=torch.int32, device="cuda")])
    q = U.queries(128, 32, D, 0)
    got = U.run_decode(more, torch.cat([q, q[:1]]), check=False)
    assert torch.equal(got[0][:128], out) and torch.equal(got[1][:128], lse)
    assert (got[0][128] == 0).all() and torch.isinf(got[1][128]).all()


def test_replayed_while_a_request_becomes_long():
    """The rule is the device's: a captured step of short requests, one of which grows."""
    c = U.Cache([5000] + [40] * 40, 2, 64, 16, seed=9)
    q, d = U.queries(41, 32, 64), c.dims(32)
    lens, ws = torch.zeros(41, dtype=torch.int32, device="cuda"), B.attn_workspace(d)
    out, lse = torch.empty_like(q), torch.empty((41, 32), device="cuda")
    go = lambda: B.moe_attn_decode(q, c.k, c.v, c.table, lens, d, out, lse, ws)  # noqa: E731
    go()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go()
    for n in (0, 30, 900, 5000, 12):
        c.lens_np = np.array([n] + [40] * 40)
        c.lens.copy_(torch.tensor(c.lens_np))
        lens.copy_(c.lens)
        g.replay()
        torch.cuda.synchronize()
        want = U.run_decode(c, q)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 7, 1), (128, 5, 1), (256, 4, 2)])
@pytest.mark.parametrize("pairs", [True, False])
def test_the_most_requests_and_groups(kind, D, Hq, Hkv, pairs):
    """The largest plan beside what the kernels keep in LDS."""
    lens = lengths(1024, D, 50)
    shared = [(r, r + 2, 16) for r in range(0, 1024, 2)] if pairs else [(r, r + 1, 16) for r in range(1024)]
    check(kind, lens, Hq, Hkv, D, shared, seed=D)
