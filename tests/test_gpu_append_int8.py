"""moe_kv_append_int8 against the oracle, bit for bit: codes and scales, what is not
written included."""
import numpy as np
import pytest
import torch

from oracle import kv_cache as K
from paper_2607_00466_amd import binding as B
from tests.kv_cache_util import Int8Cache, Rows, append_int8, bits, check_append_int8, i32

pytestmark = pytest.mark.gpu


def tables(new, held, bs, nb, seed=0, spare=1):
    """Scattered pages for held + new tokens of each request."""
    ids = list(np.random.default_rng(seed).permutation(nb))
    want = [-(-(h + n) // bs) for h, n in zip(held, new)]
    t = np.full((len(new), max(want) + spare), -1, np.int32)
    for r, w in enumerate(want):
        for i in range(w):
            t[r, i] = ids.pop()
    return t


def run(new, held, Hq, Hkv, D, rot, bs, pad_tokens=0, seed=0, q=True, pad=0, eps=1e-6, **kw):
    T = sum(new) + pad_tokens
    r = Rows(T, Hq, Hkv, D, rot, seed=seed, **kw)
    nb = sum(-(-(h + n) // bs) for h, n in zip(held, new)) + 3
    c = Int8Cache(nb, Hkv, bs, D, seed=seed + 1, pad=pad)
    start, table = np.concatenate([[0], np.cumsum(new)]), tables(new, held, bs, nb, seed)
    before = c.numpy()
    append_int8(r, c, start, table, held, q=q, eps=eps)
    check_append_int8(r, c, before, start, table, held, eps)
    if q:
        want = torch.from_numpy(r.expected("q", eps)).bfloat16()
        n = sum(new)
        assert torch.equal(bits(r.q_out.cpu()[:n]), bits(want[:n])) and (r.q_out[n:] == 7).all()
    return r, c


@pytest.mark.parametrize("D,Hq,Hkv,rot", [(64, 8, 2, 64), (128, 6, 3, 64), (256, 2, 1, 256), (128, 71, 1, 0)])
@pytest.mark.parametrize("bs", [16, 32, 128])
@pytest.mark.parametrize("fp32,interleaved,norms", [(True, False, True), (False, True, True), (False, False, False)])
def test_runs_of_every_kind(D, Hq, Hkv, rot, bs, fp32, interleaved, norms):
    # one token, none, up to a page's end, over it, whole pages, several of them
    new = [1, 0, 7, 16, bs, 2 * bs + 5, 33, 0]
    held = [0, 5, bs - 7, bs - 1, 0, 3, 2 * bs, 1]
    run(new, held, Hq, Hkv, D, rot, bs, fp32=fp32, interleaved=interleaved, norms=norms, axes=1 + fp32, seed=D + bs)


@pytest.mark.parametrize("R", [1, 63, 64, 65, 200, 1024])
def test_one_token_of_each_request(R):
    held = [(7 * r) % 40 for r in range(R)]
    run([1] * R, held, 4, 2, 64, 64, 16, seed=R)


@pytest.mark.parametrize("bs", [16, 256, 1024])
def test_a_long_prompt(bs):
    run([2500], [13], 2, 1, 64, 64, bs, seed=bs)


def test_padding_tokens_strided_pages_and_no_queries():
    run([3, 30], [14, 0], 4, 2, 128, 128, 16, pad_tokens=6, pad=32)
    run([3, 30], [14, 0], 4, 2, 128, 128, 16, pad_tokens=6, q=False)


def test_what_is_not_stored():
    """Absent pages, tokens past the table, lengths and starts out of range."""
    r = Rows(60, 2, 2, 64, 64, seed=2)
    c = Int8Cache(6, 2, 16, 64)
    table = np.array([[0, -1, 9], [1, 2, 6], [3, 4, 5]], np.int32)
    for start, lens in (([0, 20, 40, 60], [10, 30, 47]), ([0, 20, 40, 900], [-5, 10 ** 6, 16]), ([-3, -1, 30, 30], [0, 1, 48])):
        before = c.numpy()
        append_int8(r, c, start, table, lens)
        check_append_int8(r, c, before, start, table, lens)


def test_scales_zero_growing_and_not_finite():
    r = Rows(48, 1, 1, 64, 0, norms=False, seed=3)
    v = r.v.clone()
    v[0:8] = 0                      # all zeros onto a page of zeros
    v[8:16] *= 1e-20                # below what the page holds
    v[16:24] *= 2.0 ** 40           # far above it: its codes vanish
    v[24, 0, 5] = float("nan")
    v[32, 0, 6] = float("inf")
    v[40:48] = torch.full((), 1e-45)  # a scale that rounds to 0
    r.v = v
    c = Int8Cache(6, 1, 16, 64, seed=4)
    c.v_scale[0] = 0.0
    c.v_scale[5] = float("nan")
    table = np.arange(6, dtype=np.int32)[:, None]
    start, held = np.arange(0, 49, 8), [8] * 4 + [0, 8]
    before = c.numpy()
    append_int8(r, c, start, table, held)
    check_append_int8(r, c, before, start, table, held)
    s = c.v_scale[:, 0].cpu().numpy()
    assert s[0] == 0 and s[1] == before[3][1, 0] and np.isnan(s[[3, 4, 5]]).all()
    fresh = Int8Cache(1, 1, 16, 64, seed=5)
    before = fresh.numpy()
    r2 = Rows(8, 1, 1, 64, 0, norms=False, seed=3)
    r2.v = v[40:48]
    append_int8(r2, fresh, [0, 8], [[0]], [0])
    check_append_int8(r2, fresh, before, [0, 8], [[0]], [0])


def test_token_by_token_stays_within_a_step():
    """A page filled one token at a time: no value more than one step of the page's last
    scale off (half of one when written, and the halves of the growths before)."""
    r = Rows(48, 2, 2, 64, 0, norms=False, seed=6)
    r.v = (r.v * (1.3 ** torch.arange(48, device="cuda"))[:, None, None]).contiguous()
    c = Int8Cache(4, 2, 16, 64, seed=7)
    table = [[2, 0, 3]]
    one = Rows(1, 2, 2, 64, 0, norms=False, seed=6)
    for j in range(48):
        one.q, one.k, one.v = r.q[j:j + 1], r.k[j:j + 1], r.v[j:j + 1]
        append_int8(one, c, [0, 1], table, [j])
    k, ks, v, vs = c.numpy()
    for codes, scale, x in ((k, ks, r.numpy("k")), (v, vs, r.numpy("v"))):
        for j in range(48):
            page = table[0][j // 16]
            off = np.abs(codes[page, :, j % 16] * scale[page].astype(np.float64)[:, None] - x[j])
            assert (off <= scale[page][:, None] * (1 + 1e-6)).all()


def test_replayed_while_lengths_grow():
    """A step captured once and replayed: lens moves on between replays, on the device."""
    R, steps = 5, 40
    rows = [Rows(R, 4, 2, 128, 64, seed=s) for s in range(steps)]
    live = Rows(R, 4, 2, 128, 64, seed=99)
    for r in rows:  # the tables and weights of all are one's
        r.cos_np, r.sin_np, r.axis_np, r.qn_np, r.kn_np = live.cos_np, live.sin_np, live.axis_np, live.qn_np, live.kn_np
    held = np.array([0, 3, 15, 16, 30])
    c = Int8Cache(40, 2, 16, 128, seed=8)
    table = tables([steps] * R, held, 16, 40)
    k0, ks0, v0, vs0 = c.numpy()
    q, k, v = (torch.empty((R, n, 128), device="cuda") for n in (4, 2, 2))
    pos, lens, start, tab = torch.zeros((1, R), dtype=torch.int32, device="cuda"), i32(held), i32(np.arange(R + 1)), i32(table)
    d = c.dims(R, 4, table.shape[1])

    def go():
        B.moe_kv_append_int8(q, k, v, pos, live.axis, live.cos, live.sin, start, tab, lens, d, live.q_out, c.k, c.v, c.k_scale,
                             c.v_scale, live.q_norm, live.k_norm)
        lens.add_(1)

    q.fill_(1), k.fill_(1), v.fill_(1)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go()
    lens.copy_(i32(held))
    for j, r in enumerate(rows):
        for dst, src in ((q, r.q), (k, r.k), (v, r.v), (pos, r.positions)):
            dst.copy_(src)
        g.replay()
        k0, ks0 = K.append_int8(r.expected("k"), np.arange(R + 1), table, held + j, k0, ks0)
        v0, vs0 = K.append_int8(r.numpy("v"), np.arange(R + 1), table, held + j, v0, vs0)
        want = torch.from_numpy(r.expected("q")).bfloat16()
        torch.cuda.synchronize()
        assert torch.equal(bits(live.q_out.cpu()), bits(want))
    for got, want in zip(c.numpy(), (k0, ks0, v0, vs0)):
        np.testing.assert_array_equal(got, want)


def test_on_two_streams_at_once():
    calls = []
    for i in range(2):
        r, c = Rows(300, 4, 2, 128, 128, seed=i), Int8Cache(25, 2, 16, 128, seed=i)
        calls.append((r, c, c.numpy(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    table = np.arange(25, dtype=np.int32)[None]
    for r, c, _, s in calls:
        append_int8(r, c, [0, 300], table, [5], stream=s)
    for r, c, before, _ in calls:
        check_append_int8(r, c, before, [0, 300], table, [5])


@pytest.mark.parametrize("top", [1.0, 3.7e-3, 811.3, 2.0 ** -100, 1.1e-41, 3.3e38])
def test_values_at_the_borders_between_codes(top):
    """Half steps and the fp32 numbers around them: the quotient that is rounded is the
    correctly rounded one."""
    top = np.float32(top)
    scale = top * (np.float32(1) / np.float32(127))
    x = ((np.arange(0, 127) + np.float32(0.5)) * scale).astype(np.float32)
    near = [x]
    for _ in range(4):
        near += [np.nextafter(near[-1], np.float32(np.inf))]
    down = x
    for _ in range(4):
        down = np.nextafter(down, np.float32(-np.inf))
        near += [down]
    x = np.concatenate(near).astype(np.float32)
    x = np.minimum(np.concatenate([x, -x, np.full(-2 * len(x) % 64, top, np.float32)]), top)
    x[::64] = top  # every row has the largest value
    r = Rows(len(x) // 64, 1, 1, 64, 0, norms=False, seed=9)
    r.v = torch.from_numpy(x.reshape(-1, 1, 64)).cuda()
    c = Int8Cache(3, 1, 16, 64, seed=10)
    before = c.numpy()
    append_int8(r, c, [0, r.T], [[2, 0, 1]], [0])
    check_append_int8(r, c, before, [0, r.T], [[2, 0, 1]], [0])


def test_a_hundred_thousand_tokens():
    """More tokens than a 16-bit grid has, none of them normed or turned."""
    T = 100_003
    r = Rows(T, 1, 1, 64, 0, norms=False, seed=11, fp32=False)
    c = Int8Cache(-(-(T + 5) // 16) + 1, 1, 16, 64, seed=12)
    table = np.random.default_rng(0).permutation(c.nb)[None].astype(np.int32)
    before = c.numpy()
    append_int8(r, c, [0, T], table, [5])
    check_append_int8(r, c, before, [0, T], table, [5])
    assert torch.equal(bits(r.q_out), bits(r.q.contiguous()))


def test_offsets_past_2_to_31():
    """Pages whose first code lies past 2^31, where the cache is 2.3 GB."""
    nb, Hkv, bs, D = 35_200, 4, 128, 128
    r, c = Rows(300, 4, Hkv, D, 64, seed=13), Int8Cache(4, Hkv, bs, D, seed=14)
    k, v = (torch.empty((nb, Hkv, bs, D), dtype=torch.int8, device="cuda") for _ in "kv")
    ks, vs = (torch.empty((nb, Hkv), device="cuda") for _ in "kv")
    first = nb - c.nb
    k[first:], v[first:], ks[first:], vs[first:] = c.k, c.v, c.k_scale, c.v_scale
    table = np.array([[2, 0, 3]], np.int32)
    append_int8(r, c, [0, 300], table, [50])
    B.moe_kv_append_int8(r.q, r.k, r.v, r.positions, r.axis, r.cos, r.sin, i32([0, 300]), i32(table + first), i32([50]),
                         B.attn_dims(1, 4, Hkv, D, bs, 3, nb, torch.int8), r.q_out, k, v, ks, vs, r.q_norm, r.k_norm)
    for big, small in ((k, c.k), (v, c.v), (ks, c.k_scale), (vs, c.v_scale)):
        assert torch.equal(big[first:], small)
