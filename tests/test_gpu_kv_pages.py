"""moe_kv_fork and moe_kv_compact against the oracle: every byte of the caches, scales,
tables and lengths."""
import numpy as np
import pytest
import torch

from oracle import kv_cache as K
from paper_2607_00466_amd import binding as B
from tests.kv_cache_util import FP8, dev, i32

pytestmark = pytest.mark.gpu

KINDS = {"bf16": torch.bfloat16, "fp8": FP8, "int8": torch.int8}


class Pool:
    """Caches of several layers, filled with any bits; as the oracle sees them, raw."""

    def __init__(self, layers, nb, Hkv, bs, D, kind, seed=0, interleaved=False, flat=False):
        rng = np.random.default_rng(seed)
        raw = np.int16 if kind == "bf16" else np.int8
        self.kind, self.shape = kind, (layers, nb, Hkv, bs, D)
        self.caches = []
        for _ in "kv":
            x = dev(rng.integers(-128, 128, self.shape).astype(raw)).view(KINDS[kind])
            if interleaved:  # [num_blocks, layers, ...] in memory
                x = x.view(torch.uint8).transpose(0, 1).contiguous().view(KINDS[kind]).transpose(0, 1)
            self.caches.append(x[0] if flat else x)
        self.block_stride = layers * Hkv * bs * D if interleaved else 0
        self.scales = [dev(rng.random((layers, nb, Hkv)).astype(np.float32)) for _ in "kv"] if kind == "int8" else []
        if flat:
            self.scales = [s[0] for s in self.scales]

    def dims(self, R, mb):
        _, nb, Hkv, bs, D = self.shape
        return B.attn_dims(R, Hkv, Hkv, D, bs, mb, nb, KINDS[self.kind], self.block_stride)

    def numpy(self):
        raw = torch.int16 if self.kind == "bf16" else torch.int8
        caches = [c.contiguous().view(raw).cpu().numpy().reshape(self.shape) for c in self.caches]
        return caches, [s.cpu().numpy().reshape(self.shape[:3]) for s in self.scales]

    def args(self):
        return (*self.caches, *(self.scales or (None, None)))


def same(pool, want):
    caches, scales = pool.numpy()
    for a, b in zip(caches + scales, list(want[0]) + list(want[1])):
        np.testing.assert_array_equal(a, b)


def fork(pool, parent, child, page, table, lens):
    before = pool.numpy()
    t, n = i32(table), i32(lens)
    B.moe_kv_fork(i32(parent), i32(child), i32(page), t, n, pool.dims(*table.shape), *pool.args())
    torch.cuda.synchronize()
    want_t, want_n, *want = K.fork(parent, child, page, table, np.asarray(lens), *before)
    np.testing.assert_array_equal(t.cpu().numpy(), want_t)
    np.testing.assert_array_equal(n.cpu().numpy(), want_n)
    same(pool, want)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layers,Hkv,bs,D", [(1, 1, 16, 64), (3, 4, 16, 128), (5, 2, 64, 256), (48, 2, 16, 64), (2, 3, 1024, 128)])
def test_fork(kind, layers, Hkv, bs, D):
    nb = 24
    pool = Pool(layers, nb, Hkv, bs, D, kind, seed=bs)
    table = np.full((9, 4), -1, np.int32)
    lens = [0, 1, bs - 1, bs, bs + 1, 4 * bs, 0, 77, 0]
    ids = iter(np.random.default_rng(1).permutation(12))
    for r in range(6):
        for i in range(-(-lens[r] // bs)):
            table[r, i] = next(ids)
    table[6:] = [[20, 21, 22, 23]] * 3  # what is there before does not matter
    fork(pool, [1, 2, 2], [6, 7, 8], [12, 13, 14], table, lens)
    fork(pool, [3, 4, 5], [7, 8, 6], [15, 16, 17], table, lens)
    fork(pool, [0], [7], [18], table, lens)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_fork_layouts(kind):
    table, lens = np.array([[3, 1], [-1, -1]], np.int32), [21, 0]
    for kw in (dict(interleaved=True), dict(flat=True)):
        layers = 1 if "flat" in kw else 4
        fork(Pool(layers, 6, 2, 16, 128, kind, seed=2, **kw), [0], [1], [5], table, lens)


def test_fork_refuses_nothing_that_is_absent():
    """Rows and pages out of range, a child that is its parent, lengths out of range."""
    pool = Pool(2, 8, 2, 16, 64, "int8", seed=3)
    table = np.array([[0, 1, 2], [3, -1, 4], [5, 99, 4], [6, 6, 6], [7, 7, 7], [-1, -1, -1]], np.int32)
    lens = [20, 25, 25, 10 ** 6, -3, 5]
    fork(pool, [-1, 9, 0], [3, 4, 12], [6, 7, 6], table, lens)     # no such rows
    fork(pool, [0, 1], [0, 3], [6, 7], table, lens)                # itself; a parent's page that is absent
    fork(pool, [2, 0], [3, 4], [6, -1], table, lens)               # a parent's page past the cache; no page given
    fork(pool, [3, 4, 5], [0, 1, 2], [6, 7, 100], table, lens)     # a length past the table, one below 0, an absent page


def compact(pool, remap, table, in_place=False):
    before = pool.numpy()
    t = i32(table)
    out = t if in_place else torch.full_like(t, 55)
    B.moe_kv_compact(i32(remap), t, out, pool.dims(*table.shape), *pool.args())
    torch.cuda.synchronize()
    want_t, *want = K.compact(np.asarray(remap), table, *before)
    np.testing.assert_array_equal(out.cpu().numpy(), want_t)
    same(pool, want)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layers,nb,Hkv,bs,D", [(1, 1, 1, 16, 64), (3, 40, 4, 16, 128), (48, 9, 2, 16, 64), (2, 7, 2, 1024, 128), (5, 300, 1, 32, 256)])
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(kind, layers, nb, Hkv, bs, D, in_place):
    rng = np.random.default_rng(nb)
    pool = Pool(layers, nb, Hkv, bs, D, kind, seed=nb)
    live = np.flatnonzero(rng.random(nb) < 0.5)
    remap = np.full(nb, -1)
    remap[live] = live
    free = [b for b in range(len(live)) if remap[b] < 0]
    for b, to in zip([b for b in live if b >= len(live)], free):
        remap[b] = to
    table = rng.integers(-2, nb + 2, (5, 7)).astype(np.int32)
    compact(pool, remap, table, in_place)


def test_compact_frees_and_leaves_what_is_held():
    pool = Pool(2, 8, 2, 16, 64, "int8", seed=5)
    table = np.array([[0, 1, 2, 3, 4, 5, 6, 7, -1, 8, -100, 100]], np.int32)
    compact(pool, [-1] * 8, table)                       # all free
    compact(pool, list(range(8)), table)                 # nothing moves
    compact(pool, [1, 0, 3, -1, -7, 6, 99, 3 + 1], table)  # a swap is none: both are held; others move into free ones
    compact(pool, [10 ** 9, -2 ** 31, 2, 3, 0, 1, 6, 7], table)
    compact(Pool(2, 8, 2, 16, 64, "bf16", interleaved=True), [-1, -1, 2, 3, 0, 1, 6, 7], table)


def test_replayed():
    pool = Pool(3, 12, 2, 16, 128, "int8", seed=6)
    table, lens = np.array([[2, 3], [4, 5], [-1, -1], [-1, -1]], np.int32), np.array([20, 31, 0, 0])
    parent, child, page, t, n = i32([0, 1]), i32([2, 3]), i32([8, 9]), i32(table), i32(lens)
    remap, out = i32([-1, -1, 2, 3, 4, 5, -1, -1, 0, 1, -1, -1]), torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    d = pool.dims(4, 2)

    def go():
        B.moe_kv_fork(parent, child, page, t, n, d, *pool.args())
        B.moe_kv_compact(remap, t, out, d, *pool.args())

    before = pool.numpy()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go()
    for _ in range(3):
        for x, was in zip(list(pool.caches) + pool.scales, before[0] + before[1]):
            x.copy_(dev(was))
        t.copy_(i32(table)), n.copy_(i32(lens))
        g.replay()
        torch.cuda.synchronize()
        want_t, want_n, *mid = K.fork([0, 1], [2, 3], [8, 9], table, lens, *before)
        want_out, *want = K.compact(remap.cpu().numpy(), want_t, *mid)
        np.testing.assert_array_equal(out.cpu().numpy(), want_out)
        np.testing.assert_array_equal(n.cpu().numpy(), want_n)
        same(pool, want)


def test_on_side_streams():
    """Each call on a stream of its own, nothing waiting between them."""
    pools = [Pool(4, 30, 2, 16, 128, "int8", seed=i) for i in range(2)]
    table, lens = np.array([[2, 3], [4, 5], [-1, -1], [-1, -1]], np.int32), np.array([20, 31, 0, 0])
    remap = np.full(30, -1)
    remap[[2, 3, 20, 25]] = [2, 3, 0, 1]
    before = [p.numpy() for p in pools]
    args = i32([0, 1]), i32([2, 3]), i32([8, 9]), i32(table), i32(lens)
    old, out, r = i32([[2, 20], [25, 3]]), torch.zeros((2, 2), dtype=torch.int32, device="cuda"), i32(remap)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pools]
    B.moe_kv_fork(*args, pools[0].dims(4, 2), *pools[0].args(), stream=streams[0])
    B.moe_kv_compact(r, old, out, pools[1].dims(2, 2), *pools[1].args(), stream=streams[1])
    for s in streams:
        s.synchronize()
    want_t, want_n, *want = K.fork([0, 1], [2, 3], [8, 9], table, lens, *before[0])
    np.testing.assert_array_equal(args[3].cpu().numpy(), want_t)
    same(pools[0], want)
    want_out, *want = K.compact(remap, np.array([[2, 20], [25, 3]]), *before[1])
    np.testing.assert_array_equal(out.cpu().numpy(), want_out)
    same(pools[1], want)


def test_no_layer_and_no_page():
    """The tables alone; and a cache without a page, of which everything is absent."""
    for layers, nb in ((0, 6), (2, 0)):
        d = B.attn_dims(2, 2, 2, 64, 16, 2, nb, torch.bfloat16)
        k = torch.zeros((layers, nb, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
        t, n = i32([[4, 3], [-1, -1]]), i32([20, 0])
        B.moe_kv_fork(i32([0]), i32([1]), i32([5]), t, n, d, k, k.clone())
        assert t.tolist() == [[4, 3], [4, 5 if nb else -1]] and n.tolist() == [20, 20]
        B.moe_kv_compact(i32([-1, -1, -1, 0, 1, 2][:nb]), t, t, d, k, k.clone())
        assert t.tolist() == ([[1, 0], [1, 2]] if nb else [[-1, -1], [-1, -1]])


def test_offsets_past_2_to_31():
    """A page of the last of eight layers, past 2^31 codes: everything else stays."""
    layers, nb, Hkv, bs, D = 8, 36_000, 4, 16, 128
    caches = [torch.randint(-128, 128, (layers, nb, Hkv, bs, D), dtype=torch.int8, device="cuda") for _ in "kv"]
    scales = [torch.rand((layers, nb, Hkv), device="cuda") for _ in "kv"]
    was = [x.clone() for x in caches + scales]
    d = B.attn_dims(2, 4, Hkv, D, bs, 2, nb, torch.int8)
    remap = torch.full((nb,), -1, dtype=torch.int32, device="cuda")
    remap[nb - 1], remap[7], remap[100] = nb - 2, 7, nb - 3
    t = i32([[nb - 1, 7], [100, -1]])
    B.moe_kv_compact(remap, t, t, d, *caches, *scales)
    assert t.tolist() == [[nb - 2, 7], [nb - 3, -1]]
    for x, w in zip(caches + scales, was):
        w[:, nb - 2], w[:, nb - 3] = w[:, nb - 1].clone(), w[:, 100].clone()
        assert torch.equal(x, w)
    n = i32([21, 0])
    B.moe_kv_fork(i32([0]), i32([1]), i32([nb - 5]), t, n, d, *caches, *scales)
    assert t.tolist() == [[nb - 2, 7], [nb - 2, nb - 5]] and n.tolist() == [21, 21]
    for x, w in zip(caches, was):
        w[:, nb - 5, :, :5] = w[:, 7, :, :5].clone()
        assert torch.equal(x, w)
    for x, w in zip(scales, was[2:]):
        w[:, nb - 5] = w[:, 7].clone()
        assert torch.equal(x, w)


def test_a_tensor_on_another_device_is_named(monkeypatch):
    """Kernels run on the current device: a cache elsewhere is refused before the launch."""
    pool = Pool(1, 4, 2, 16, 64, "bf16", flat=True)
    t = i32([[0, 1]])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="k_cache: is on cuda:0, and the current device is cuda:1"):
        B.moe_kv_compact(i32([0, 1, 2, 3]), t, t, pool.dims(1, 2), *pool.args())
