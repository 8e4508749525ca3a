"""moe_attn_decode over pages of 8-bit integers, against the oracle within the bounds
that hold for the other caches (codes enter the products exactly, and a page's scale is
one more rounding of a score and of a weight)."""
import numpy as np
import pytest
import torch

from paper_2607_00466_amd import binding as B
from tests import attention_util as U

pytestmark = pytest.mark.gpu


class Cache(U.Cache):
    """As for the other types: what no request has cached holds any code, and pages of
    which nothing is cached have scales that are no number."""

    def __init__(self, lens, Hkv, D, bs, seed=0, **kw):
        super().__init__(lens, Hkv, D, bs, seed=seed, **kw)
        rng = np.random.default_rng(seed + 100)
        stride = self.k.stride(0)
        used = np.isfinite(self.k_np[:, 0, :, 0])  # [nb, bs]: garbage is not finite, or huge
        used &= np.abs(self.k_np[:, 0]).max(-1) < 1e30
        self.scales = []
        for which in ("k", "v"):
            x = getattr(self, which + "_np")
            x = np.where(used[:, None, :, None], x, 0.0)
            scale = (np.abs(x).max((-1, -2)) / 127 * rng.uniform(1, 2, x.shape[:2])).astype(np.float32)
            codes = np.rint(x / np.where(scale > 0, scale, 1)[:, :, None, None]).astype(np.int8)
            codes[~np.broadcast_to(used[:, None, :, None], codes.shape)] = rng.integers(-128, 128)
            scale[~used.any(-1)] = np.nan
            setattr(self, which + "_np", codes * scale.astype(np.float64)[:, :, None, None])
            setattr(self, which, self._place(torch.from_numpy(codes), stride))
            setattr(self, which + "_scale", torch.from_numpy(scale).cuda())

    def dims(self, Hq):
        d = super().dims(Hq)
        d.kv_type = B.MOE_KV_INT8
        return d


def check(lens, Hq, Hkv, D, bs=16, shared=(), sinks=False, window=0, seed=0, **kw):
    c = Cache(lens, Hkv, D, bs, seed=seed, shared=shared, **kw)
    q = U.queries(len(lens), Hq, D, seed)
    s = torch.randn(Hq, generator=torch.Generator().manual_seed(seed)).cuda() * 3 if sinks else None
    out, lse = U.run_decode(c, q, shared, s, window)
    return c, q, out, lse


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("bs", [16, 64])
def test_lengths_around_every_tile(D, bs):
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 255, 256, 257, 500, 513]
    check(lens, 8, 2, D, bs, seed=D)
    check(lens, 8, 2, D, bs, sinks=True, seed=D + 1, pad=64)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (5, 1), (16, 1), (17, 1), (71, 1), (64, 8), (20, 4)])
def test_head_groups(Hq, Hkv):
    check([3, 100, 190], Hq, Hkv, 64)
    check([3, 100, 190], Hq, Hkv, 128, window=50)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_groups(D):
    shared = [(0, 3, 64), (3, 4, 100), (4, 9, 200), (10, 12, 33)]
    lens = [70, 64, 300, 100, 200, 201, 0, 455, 233, 12, 40, 33, 500]
    check(lens, 8, 2, D, 16, shared, seed=D)
    check(lens, 8, 2, D, 32, shared, sinks=True, seed=D + 1)
    check([1100 + r for r in range(20)], 16, 2, D, 16, [(0, 20, 1090)], seed=D + 2)


@pytest.mark.parametrize("window", [1, 15, 16, 17, 40, 128, 129, 1000])
def test_windows(window):
    """Pages before the window: their scales do not count either."""
    lens = [0, 1, 16, 33, 130, 400]
    c, q, out, lse = check(lens, 8, 2, 128, 16, window=window)
    for r, n in enumerate(lens):
        for b in range(max(0, n - window) // 16):
            c.k_scale[int(c.table_np[r, b])] = c.v_scale[int(c.table_np[r, b])] = float("nan")
    again = U.run_decode(c, q, window=window, check=False)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


def test_absent_pages():
    c = Cache([100, 64, 300, 40], 2, 128, 16, seed=3)
    c.table_np[0, 2] = -1
    c.table_np[1, :] = c.nb
    c.table_np[2, [0, 5, 18]] = [-7, 10 ** 6, -1]
    c.table = torch.from_numpy(c.table_np).cuda()
    U.run_decode(c, U.queries(4, 8, 128))


def test_a_holey_prefix():
    c = Cache([230, 240, 250], 2, 128, 16, seed=4, shared=[(0, 3, 220)])
    c.table_np[0, [1, 6, 7]] = -1
    c.table = torch.from_numpy(c.table_np).cuda()
    U.run_decode(c, U.queries(3, 8, 128), [(0, 3, 220)])


def test_scales_that_count_when_they_are_nan():
    """In a page of which a slot is visible: NaN for that request and kv head alone."""
    for which in ("k_scale", "v_scale"):
        c = Cache([100, 50], 2, 64, 16, seed=5)
        getattr(c, which)[int(c.table_np[0, 3]), 1] = float("nan")
        out, lse = U.run_decode(c, U.queries(2, 8, 64), check=False)
        assert out[0, 4:].isnan().all() and out[0, :4].isfinite().all() and out[1].isfinite().all()
        assert lse[0, 4:].isnan().all() == (which == "k_scale")


def test_scales_of_zero_and_far_apart():
    """Pages of zeros, and scales 2^60 apart: the bounds are of the largest rows."""
    c = Cache([200, 130], 1, 128, 16, seed=6)
    k, v = c.k_scale.clone(), c.v_scale.clone()
    for i, b in enumerate(c.table_np[0, :12]):
        k[int(b)] *= [0.0, 2.0 ** -60, 1.0][i % 3]
        v[int(b)] *= [1.0, 0.0, 2.0 ** -60, 2.0 ** 30][i % 4]
    c.k_scale, c.v_scale = k, v
    c.k_np = c.k.cpu().numpy() * k.double().cpu().numpy()[:, :, None, None]
    c.v_np = c.v.cpu().numpy() * v.double().cpu().numpy()[:, :, None, None]
    U.run_decode(c, U.queries(2, 4, 128))


def test_many_long_requests_and_splits():
    check([4000 + 37 * r for r in range(6)], 16, 2, 128, 16, seed=7)
    check([9000], 8, 1, 64, 1024, seed=8)


def test_offsets_past_2_to_31():
    """Pages whose first element lies past 2^31, where the cache is 2.3 GB."""
    nb, Hkv, bs, D = 35_200, 4, 128, 128
    c = Cache([300, 17], Hkv, D, bs, seed=9)
    k, v = (torch.empty((nb, Hkv, bs, D), dtype=torch.int8, device="cuda") for _ in "kv")
    ks, vs = (torch.full((nb, Hkv), float("nan"), device="cuda") for _ in "kv")
    first = nb - c.nb
    k[first:], v[first:], ks[first:], vs[first:] = c.k, c.v, c.k_scale, c.v_scale
    table = torch.where(c.table >= 0, c.table + first, -1)
    q = U.queries(2, 8, D)
    want = U.run_decode(c, q)
    d = B.attn_dims(2, 8, Hkv, D, bs, c.max_blocks, nb, torch.int8)
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    B.moe_attn_decode(q, k, v, table, c.lens, d, out, lse, B.attn_workspace(d), k_scale=ks, v_scale=vs)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_replays_while_lengths_grow():
    c = Cache([300, 290], 2, 128, 16, seed=10)
    q, d = U.queries(2, 8, 128), c.dims(8)
    lens, ws = torch.zeros(2, dtype=torch.int32, device="cuda"), B.attn_workspace(d)
    out, lse = torch.empty_like(q), torch.empty((2, 8), device="cuda")
    go = lambda: B.moe_attn_decode(q, c.k, c.v, c.table, lens, d, out, lse, ws, k_scale=c.k_scale, v_scale=c.v_scale)  # noqa: E731
    go()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go()
    for a, b in ((0, 1), (16, 17), (128, 250), (300, 290)):
        lens.copy_(torch.tensor([a, b]))
        g.replay()
        got = out.clone(), lse.clone()
        go()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], lse)
