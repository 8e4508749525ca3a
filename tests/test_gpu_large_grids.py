"""Launches of more threads than 32 bits count: every workgroup runs.  (Nearly all of them
find nothing to do, and most of the memory is never read or written.)"""
import numpy as np
import pytest
import torch

from oracle import kv_cache as K
from paper_2607_00466_amd import binding as B
from tests.kv_cache_util import i32

pytestmark = pytest.mark.gpu

ROW = 1 << 24  # workgroups of 256 threads


@pytest.fixture(autouse=True)
def alone():
    """Tens of gigabytes a test: none of them stay."""
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_compact_a_pool_of_many_pages():
    nb = ROW + 1000
    caches = [torch.empty((nb, 1, 16, 64), dtype=torch.int8, device="cuda") for _ in "kv"]
    scales = [torch.empty((nb, 1), device="cuda") for _ in "kv"]
    moves = {nb - 1: 3, nb - 500: ROW + 7, 77: 12}
    remap = torch.full((nb,), -1, dtype=torch.int32, device="cuda")
    remap[5] = 5
    for i, (b, to) in enumerate(moves.items()):
        remap[b] = to
        for n, t in enumerate(caches + scales):
            t[b], t[to] = 10 * i + n + 1, 0
    table = i32([[nb - 1, 5, -1, nb - 500], [77, 9, nb, 3]])
    B.moe_kv_compact(remap, table, table, B.attn_dims(2, 1, 1, 64, 16, 4, nb, torch.int8), *caches, *scales)
    assert table.tolist() == [[3, 5, -1, ROW + 7], [12, -1, -1, -1]]
    for i, to in enumerate(moves.values()):
        for n, t in enumerate(caches + scales):
            assert (t[to] == 10 * i + n + 1).all()


@pytest.mark.parametrize("queries", [False, True])
def test_append_a_million_tokens_of_many_heads(queries):
    """Two requests of 2^19 tokens, of whose pages a few are there."""
    T, Hkv, D, bs, mb = 1 << 20, 256, 64, 32, 1 << 14
    x = torch.empty((T, Hkv, D), dtype=torch.bfloat16, device="cuda")  # keys, values and queries alike
    q_out = torch.empty((T, Hkv, D), dtype=torch.bfloat16, device="cuda") if queries else None
    table, at = np.full((2, mb), -1, np.int32), {(0, 0): 2, (0, mb - 1): 0, (1, 1): 5, (1, mb - 1): 3}
    rng, rows = np.random.default_rng(0), {}
    for (r, j), page in at.items():
        table[r, j] = page
        first = r * (T // 2) + j * bs
        x[first:first + bs] = torch.from_numpy(rng.standard_normal((bs, Hkv, D)).astype(np.float32)).cuda()
        rows[page] = first
    codes = [torch.full((6, Hkv, bs, D), 99, dtype=torch.int8, device="cuda") for _ in "kv"]
    scales = [torch.full((6, Hkv), 7.0, device="cuda") for _ in "kv"]
    none = torch.zeros((1, 0), device="cuda")
    B.moe_kv_append_int8(x if queries else None, x, x, torch.zeros((1, T), dtype=torch.int32, device="cuda"), i32([]), none, none,
                         i32([0, T // 2, T]), i32(table), i32([0, 0]), B.attn_dims(2, Hkv, Hkv, D, bs, mb, 6, torch.int8), q_out,
                         *codes, *scales)
    for c, s in zip(codes, scales):
        for page, first in rows.items():
            new = x[first:first + bs].float().cpu().numpy()
            want = K.append_int8(new, [0, bs], [[0]], [0], np.zeros((1, Hkv, bs, D), np.int8), np.zeros((1, Hkv), np.float32))
            np.testing.assert_array_equal(c[page].cpu().numpy(), want[0][0])
            np.testing.assert_array_equal(s[page].cpu().numpy(), want[1][0])
        assert (c[[1, 4]] == 99).all() and (s[[1, 4]] == 7).all()
    if queries:
        for first in rows.values():
            assert torch.equal(q_out[first:first + bs], x[first:first + bs])


def test_capture_of_many_picks():
    """2^32 + 2^23 picks, of which two tokens' are in a block."""
    layers, T, K, E = 513, 1 << 20, 8, 32
    ids = torch.empty((layers, T, K), dtype=torch.int32, device="cuda")
    block = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    few = torch.randint(0, E, (layers, 2, K), dtype=torch.int32, device="cuda")
    tokens, blocks = [3, T - 1], i32([2, 0])
    ids[:, tokens], block[tokens] = few, blocks
    L = 516
    got, want = (torch.zeros((3, L, E), dtype=torch.int8, device="cuda") for _ in "gw")
    B.moe_sig_capture(ids, block, 2, L, E, got)
    B.moe_sig_capture(few, blocks, 2, L, E, want)
    assert torch.equal(got, want) and int(want.sum()) == 2 * layers * K


def test_pack_large_experts():
    """A layer's up projections of 2^35 values and more: the last expert's as when it is
    packed alone."""
    E, I, H = 129, 8192, 16384
    w = torch.empty((E, I, H), dtype=torch.bfloat16, device="cuda")  # w1 and w3 alike
    w[[0, E - 1]] = torch.randint(-2 ** 15, 2 ** 15, (2, I, H), dtype=torch.int16, device="cuda").view(torch.bfloat16)
    got = B.moe_pack_up_weights(w, w).view(torch.int16)
    for e in (0, E - 1):
        assert torch.equal(got[e:e + 1], B.moe_pack_up_weights(w[e:e + 1], w[e:e + 1]).view(torch.int16))


def test_pack_large_mxfp4_experts():
    E, I, H = 257, 16384, 16384
    c = torch.empty((E, I, H // 2), dtype=torch.uint8, device="cuda")
    s = torch.empty((E, I, H // 32), dtype=torch.uint8, device="cuda")
    for t in (c, s):
        t[[0, E - 1]] = torch.randint(0, 256, (2, *t.shape[1:]), dtype=torch.uint8, device="cuda")
    got = [t.view(E, -1) for t in B.moe_pack_mxfp4_up((c, s), (c, s))]
    for e in (0, E - 1):
        one = c[e:e + 1], s[e:e + 1]
        for a, b in zip(got, B.moe_pack_mxfp4_up(one, one)):
            assert torch.equal(a[e], b)
