"""GPU tests of the attention calls against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import attention as A
from paper_2607_00466_amd import binding as B
from tests import attention_util as U
from tests import gpu_util as G

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------- append

def _tables(rot, max_pos=64):
    f = 1e4 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / max(rot, 1))
    a = torch.arange(max_pos, dtype=torch.float64)[:, None] * f
    return a.cos().float(), a.sin().float()


@pytest.mark.parametrize("T,Hq,Hkv,D,rot,axes,interleaved,fp8,dtype,bs,fused", [
    (1, 1, 1, 64, 64, 1, False, False, torch.bfloat16, 16, False),
    (3, 32, 4, 128, 128, 1, False, False, torch.bfloat16, 16, True),
    (65, 8, 8, 64, 32, 3, True, True, torch.bfloat16, 16, True),
    (33, 5, 5, 128, 16, 2, False, True, torch.float32, 16, True),
    (40, 10, 2, 256, 256, 3, True, False, torch.float32, 32, False),
    (19, 6, 3, 256, 128, 8, False, True, torch.float32, 64, True),
    (7, 4, 2, 64, 0, 1, False, False, torch.bfloat16, 16, False),
])
def test_append(T, Hq, Hkv, D, rot, axes, interleaved, fp8, dtype, bs, fused):
    G.say(f"case: append T={T} heads {Hq}/{Hkv} D={D} rot={rot} axes={axes} interleaved={interleaved} fp8={fp8} {dtype}")
    rng = np.random.default_rng(T)
    g = torch.Generator().manual_seed(T)
    rows = torch.randn((T, Hq + 2 * Hkv, D), generator=g).to(dtype).cuda()
    rows[0, -1, 0] = 1e5  # saturates e4m3
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    cos, sin = _tables(rot)
    pos = torch.from_numpy(rng.integers(0, 64, (axes, T)).astype(np.int32))
    axis = torch.from_numpy(rng.integers(0, axes, rot // 2).astype(np.int32))
    nb = -(-T // bs) + 2
    slots = torch.from_numpy(rng.permutation(nb * bs)[:T].astype(np.int32))
    if T > 4:
        slots[2], slots[4] = -1, nb * bs + 5  # dropped: no slot, and a page past the cache
    d = B.attn_dims(0, Hq, Hkv, D, bs, 1, nb, U.FP8 if fp8 else torch.bfloat16, Hkv * bs * D + 32)
    caches = [U.Cache._place(torch.full((nb, Hkv, bs, D), 7.0).to(U.FP8 if fp8 else torch.bfloat16), d.block_stride)
              for _ in "kv"]
    scales = [torch.from_numpy(rng.uniform(0.5, 2, Hkv).astype(np.float32)).cuda() if fp8 else None for _ in "kv"]
    q_out = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
    B.moe_kv_append(q, k, v, pos.cuda(), axis.cuda(), cos.cuda(), sin.cuda(), slots.cuda(), d, q_out, *caches, *scales,
                    interleaved=interleaved)
    torch.cuda.synchronize()

    def fp32(x):
        """The definition in fp32, each product and sum rounded."""
        x = x.float().cpu().clone()
        at = pos.long()[axis.long()].T
        c, s = cos[at, torch.arange(rot // 2)][:, None], sin[at, torch.arange(rot // 2)][:, None]
        i = torch.arange(rot // 2)
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        a, b = x[..., lo], x[..., hi]
        ac, bs_, bc, as_ = a * c, b * s, b * c, a * s
        x[..., lo], x[..., hi] = ac - bs_, bc + as_
        return x

    def stored(x, scale):
        if not fp8:
            return x.to(torch.bfloat16).float()
        return (x / scale.cpu()[:, None]).clamp(-448, 448).to(U.FP8).float()

    assert torch.equal(q_out.cpu(), fp32(q).to(torch.bfloat16))
    exact = A.rotate(q.double().cpu().numpy(), pos.numpy(), axis.numpy(), cos.numpy(), sin.numpy(), interleaved)
    # three fp32 roundings of terms that a pair's length bounds, then bf16's
    big = np.abs(rows[:, :Hq].double().cpu().numpy()).max(-1, keepdims=True) * 1.5
    assert (np.abs(q_out.double().cpu().numpy() - exact) <= 1.01 * U.U_BF16 * np.abs(exact) + 4 * U.U_FP32 * big).all()
    for got, x, scale in ((caches[0], fp32(k), scales[0]), (caches[1], v.float().cpu(), scales[1])):
        want = torch.full((nb, Hkv, bs, D), 7.0)
        for t in range(T):
            s = int(slots[t])
            if 0 <= s < nb * bs:
                want[s // bs, :, s % bs] = stored(x[t:t + 1], scale)[0]
        assert torch.equal(got.float().cpu(), want)


@pytest.mark.parametrize("T,axes,interleaved,fp8", [(3001, 1, False, False), (2049, 3, True, True)])
def test_append_prompts(T, axes, interleaved, fp8):
    # tokens enough for a thread to turn several heads
    G.say(f"case: append of a prompt of {T}, {axes} axes, interleaved={interleaved} fp8={fp8}")
    Hq, Hkv, D, rot, bs = 33, 3, 128, 96, 16
    g = torch.Generator(device="cuda").manual_seed(T)
    rows = torch.randn((T, Hq + 2 * Hkv, D), device="cuda", generator=g)
    cos, sin = (x.cuda() for x in _tables(rot, 5000))
    pos = torch.randint(0, 5000, (axes, T), device="cuda", generator=g, dtype=torch.int32)
    axis = (torch.arange(rot // 2, device="cuda") * axes // (rot // 2)).to(torch.int32)  # its sections end inside a chunk
    nb = -(-T // bs) + 1
    slots = torch.randperm(nb * bs, device="cuda", generator=g)[:T].to(torch.int32)
    dtype = U.FP8 if fp8 else torch.bfloat16
    caches = [torch.zeros((nb, Hkv, bs, D), device="cuda").to(dtype) for _ in "kv"]
    scale = torch.linspace(0.01, 2, Hkv, device="cuda") if fp8 else None
    q_out = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
    B.moe_kv_append(rows[:, :Hq], rows[:, Hq:-Hkv], rows[:, -Hkv:], pos, axis, cos, sin, slots,
                    B.attn_dims(0, Hq, Hkv, D, bs, 1, nb, dtype), q_out, *caches, scale, scale, interleaved=interleaved)
    at = pos.long()[axis.long()].T
    i = torch.arange(rot // 2, device="cuda")
    c, s = cos[at, i][:, None], sin[at, i][:, None]
    lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    turned = rows[:, :-Hkv].clone()
    a, b = turned[..., lo], turned[..., hi]
    ac, bs_, bc, as_ = a * c, b * s, b * c, a * s
    turned[..., lo], turned[..., hi] = ac - bs_, bc + as_
    assert torch.equal(q_out, turned[:, :Hq].bfloat16())
    for cache, x in zip(caches, (turned[:, Hq:], rows[:, -Hkv:])):
        want = (x / scale[:, None]).clamp(-448, 448).to(dtype) if fp8 else x.to(dtype)
        got = cache.float()[slots.long() // bs, :, slots.long() % bs]
        assert torch.equal(got, want.float())


def test_append_positions_outside_and_keys_alone():
    G.say("case: append, positions outside the table; keys and values alone; T = 0")
    cos, sin = (t.cuda() for t in _tables(64))
    k = torch.randn((3, 1, 64), device="cuda")
    d = B.attn_dims(0, 2, 1, 64, 16, 1, 1)
    kc, vc = (torch.zeros((1, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    i32 = dict(dtype=torch.int32, device="cuda")
    axis = torch.zeros(32, **i32)
    axis[5] = 1  # an axis that is not there
    B.moe_kv_append(None, k, k, torch.tensor([[0, 64, -1]], **i32), axis, cos, sin, torch.tensor([0, 1, 2], **i32), d, None,
                    kc, vc)
    torch.cuda.synchronize()
    bad = torch.zeros(64, dtype=torch.bool, device="cuda")
    bad[[5, 37]] = True
    assert torch.equal(kc[0, 0, 0].isnan(), bad)
    assert kc[0, 0, 1:3].isnan().all() and not kc[0, 0, 3:].any()
    assert torch.equal(vc[0, 0, :3], k[:, 0].bfloat16())
    e = torch.empty((0, 1, 64), device="cuda")
    B.moe_kv_append(None, e, e, torch.empty((1, 0), **i32), axis, cos, sin, torch.empty(0, **i32), d, None, kc, vc)


# ----------------------------------------------------------------------------- decode

DECODE = [
    # lens, Hq, Hkv, D, bs, shared, fp8, window, sinks
    ([0], 1, 1, 64, 16, (), False, 0, False),
    ([0, 1], 2, 1, 128, 16, (), False, 0, True),
    ([1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 0], 8, 2, 128, 16, (), False, 0, False),
    ([127, 128, 129, 255, 256, 257, 1000], 32, 4, 128, 16, (), False, 0, False),
    ([1, 130, 700], 32, 4, 128, 32, (), True, 0, True),
    ([5, 400, 129], 64, 8, 64, 64, (), False, 128, True),
    ([33, 1029], 64, 8, 64, 16, (), True, 0, False),
    ([300, 77], 7, 1, 128, 32, (), False, 0, False),     # 7 heads a kv head
    ([300, 77], 20, 4, 64, 16, (), False, 0, False),     # 5
    ([260, 31], 32, 1, 128, 16, (), False, 0, False),    # 32: two tiles of rows
    ([260, 31], 25, 1, 64, 16, (), True, 0, True),       # 25
    ([260, 31], 71, 1, 64, 16, (), False, 0, False),     # 71: several tiles
    ([513, 64, 2], 16, 2, 256, 16, (), False, 0, False),
    ([513, 64, 2], 16, 2, 256, 256, (), True, 100, True),
    ([6000, 3], 8, 1, 128, 1024, (), False, 0, False),
    ([9000], 4, 4, 64, 16, (), False, 0, True),
    # shared prefixes: whole pages, ends inside a page, longer than a member, an empty member
    ([80, 64, 70, 65], 8, 1, 128, 16, ((0, 4, 64),), False, 0, False),
    ([300, 257, 700, 256, 290], 32, 4, 128, 16, ((0, 5, 256),), False, 0, True),
    ([300, 257, 700, 290, 290], 8, 2, 64, 16, ((1, 4, 250),), True, 0, False),
    ([80, 0, 70, 30, 5], 8, 1, 128, 16, ((0, 5, 64),), False, 0, False),
    ([200] * 9 + [333] * 8, 16, 4, 64, 32, ((0, 9, 192), (10, 17, 320)), False, 0, False),
    ([140 + i for i in range(40)], 8, 1, 128, 16, ((0, 40, 128),), False, 0, False),
    ([530 + 3 * i for i in range(37)], 16, 2, 256, 16, ((0, 37, 512),), True, 0, True),
    ([600, 640, 800], 5, 1, 128, 16, ((0, 2, 592),), False, 0, False),
    ([90, 95, 99], 8, 2, 64, 16, ((0, 3, 64),), False, 20, False),  # a window: nothing is shared
    ([1100 + i for i in range(70)], 32, 4, 128, 16, ((0, 70, 1088),), False, 0, False),
    # prefixes of several look-up windows, rows that leave row waves idle
    ([2600, 2501, 2550, 2500], 20, 4, 64, 64, ((0, 4, 2500),), True, 0, True),
    ([3100, 3201, 3150], 16, 2, 256, 16, ((0, 3, 3100),), False, 0, False),
    ([2100] * 5, 48, 1, 128, 16, ((0, 5, 2048),), False, 0, False),
]


@pytest.mark.parametrize("lens,Hq,Hkv,D,bs,shared,fp8,window,sinks", DECODE)
def test_decode(lens, Hq, Hkv, D, bs, shared, fp8, window, sinks):
    G.say(f"case: decode lens={lens[:8]} heads {Hq}/{Hkv} D={D} bs={bs} shared={shared} fp8={fp8} window={window}")
    # members of a group keep no pages of the prefix (a window reads its own rows)
    cache = U.Cache(lens, Hkv, D, bs, fp8, seed=len(lens), shared=() if window else shared, max_blocks=-(-max(lens + [1]) // bs) + 1)
    s = torch.randn(Hq, device="cuda") if sinks else None
    U.run_decode(cache, U.queries(len(lens), Hq, D), shared, s, window)


@pytest.mark.parametrize("fp8", [False, True])
def test_decode_large_batch_of_many_groups(fp8):
    G.say(f"case: decode of 300 requests, groups of 1 to 40, fp8={fp8}")
    rng = np.random.default_rng(3)
    shared, at = [], 2
    while at < 290:
        n = int(rng.integers(1, 41))
        shared.append((at, min(300, at + n), int(rng.integers(0, 6)) * 16))
        at += n
    lens = [int(x) for x in rng.integers(0, 150, 300)]
    for s, e, t in shared:
        for r in range(s, e):
            lens[r] += t
    # a page that a short member reads through the first one has to be there
    cache = U.Cache(lens, 2, 64, 16, fp8, seed=9, shared=shared)
    U.run_decode(cache, U.queries(300, 8, 64), shared)


@pytest.mark.parametrize("D,fp8", [(64, True), (256, False)])
def test_decode_most_requests_and_groups(D, fp8):
    G.say(f"case: decode of 1024 requests in 512 groups of two, D={D}: the largest plan")
    rng = np.random.default_rng(D)
    lens = [int(x) for x in rng.integers(0, 70, 1024)]
    shared = []
    for s in range(0, 1024, 2):
        n = 16 * int(rng.integers(0, 3))
        shared.append((s, s + 2, n))
        lens[s] += n
        lens[s + 1] += n
    cache = U.Cache(lens, 1, D, 16, fp8, seed=D, shared=shared)
    U.run_decode(cache, U.queries(1024, 2, D), shared)


def test_decode_peaked_and_flat_scores():
    G.say("case: decode, scores of several hundred; all keys alike; scale 0 and negative")
    cache = U.Cache([700, 40], 2, 128, 16, seed=1, amp=4.0)
    q = U.queries(2, 8, 128, amp=8.0)
    U.run_decode(cache, q)
    U.run_decode(cache, q, scale=0.0)
    U.run_decode(cache, q, scale=-0.01)


def test_decode_absent_pages_and_lengths_past_the_table():
    G.say("case: decode, absent pages, a length past the table, a negative one")
    cache = U.Cache([200, 64, 64, 112], 2, 64, 16, seed=2, max_blocks=13)  # 112: whole pages
    cache.table_np[0, 3], cache.table_np[0, 7], cache.table_np[1, :4] = -5, cache.nb + 4, 1 << 30
    cache.table.copy_(torch.from_numpy(cache.table_np))
    cache.lens_np = np.array([200, 64, -3, 5000])
    cache.lens.copy_(torch.from_numpy(cache.lens_np))
    U.run_decode(cache, U.queries(4, 4, 64))


def test_decode_interleaved_caches_and_offsets_past_32_bits():
    G.say("case: decode, keys and values of one allocation, element offsets past 2^32")
    Hkv, bs, D, nb = 2, 16, 128, 40
    lens = [333, 129]
    cache = U.Cache(lens, Hkv, D, bs, seed=4, spare=nb - 30)
    dense = Hkv * bs * D
    stride = (1 << 32) // (cache.nb - 2) // 32 * 32 + 2 * dense
    buf = torch.empty(cache.nb * stride, dtype=torch.bfloat16, device="cuda")
    k = torch.as_strided(buf, cache.k.shape, (stride, bs * D, D, 1))
    v = torch.as_strided(buf, cache.k.shape, (stride, bs * D, D, 1), dense)
    k.copy_(cache.k), v.copy_(cache.v)
    cache.k, cache.v, cache.block_stride = k, v, stride
    U.run_decode(cache, U.queries(2, 8, D))


def test_decode_is_the_same_twice_on_streams_and_in_graphs():
    G.say("case: decode, run twice, on a side stream, in a graph with changing lengths")
    lens = [700 + 13 * i for i in range(12)]
    shared = ((0, 12, 640),)
    cache = U.Cache(lens, 4, 128, 16, seed=5, shared=shared, max_blocks=64)
    q = U.queries(12, 32, 128)
    d = cache.dims(32)
    ws = B.attn_workspace(d)
    first = U.run_decode(cache, q, shared, ws=ws)
    again = U.run_decode(cache, q, shared, ws=ws)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = U.run_decode(cache, q, shared, ws=ws, stream=side)
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    # a graph reads lengths and groups on the device
    gs, pl, _, _ = U.groups_of(shared, 12)
    out, lse = torch.empty_like(first[0]), torch.empty_like(first[1])
    call = lambda: B.moe_attn_decode(q, cache.k, cache.v, cache.table, cache.lens, d, out, lse, ws, gs, pl)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        cache.lens.copy_(torch.tensor([n - 17 * step for n in lens], dtype=torch.int32))
        pl.fill_(640 - 16 * step)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        out.fill_(0)
        call()
        torch.cuda.synchronize()
        assert torch.equal(out, got[0]) and torch.equal(lse, got[1])


# ----------------------------------------------------------------------------- weights

WEIGHTS = [
    ([0, 1], 2, 1, 128, 16, (), False),
    ([1, 15, 16, 17, 33, 64, 65, 130, 300], 32, 4, 128, 16, (), False),
    ([140, 70], 7, 1, 64, 16, (), True),
    ([140, 70], 10, 2, 64, 32, (), False),
    ([140, 70], 40, 1, 128, 16, (), False),
    ([90], 4, 4, 256, 16, (), True),
    ([80, 64, 70, 65], 8, 1, 128, 16, ((0, 4, 64),), False),
    ([80, 0, 70, 30, 5], 6, 2, 64, 16, ((0, 5, 60),), True),
    ([140 + i for i in range(20)], 16, 2, 64, 16, ((0, 20, 128),), False),
    ([150 + i for i in range(9)], 5, 1, 128, 16, ((1, 9, 144),), False),
    ([150 + i for i in range(5)], 24, 1, 128, 16, ((0, 4, 144),), False),
    ([40, 50, 45], 3, 3, 256, 16, ((0, 3, 32),), False),
]


@pytest.mark.parametrize("lens,Hq,Hkv,D,bs,shared,fp8", WEIGHTS)
def test_weights(lens, Hq, Hkv, D, bs, shared, fp8):
    G.say(f"case: weights lens={lens[:8]} heads {Hq}/{Hkv} D={D} bs={bs} shared={shared} fp8={fp8}")
    cache = U.Cache(lens, Hkv, D, bs, fp8, seed=len(lens) + 1, shared=shared, max_blocks=-(-max(lens) // bs) + 1)
    R = len(lens)
    q = U.queries(R, Hq, D)
    _, lse = U.run_decode(cache, q, shared)
    gs, pl, gs_np, pl_np = U.groups_of(shared, R)
    d, scale = cache.dims(Hq), D ** -0.5
    w_in = torch.rand((R, Hkv, cache.N), device="cuda")
    e = U.score_bound(q, cache, scale)
    for given, target in ((w_in, torch.full_like(w_in, -2.0)), (None, torch.full_like(w_in, -2.0)), (w_in.clone(), None)):
        in_place = target is None
        target = given if in_place else target
        before = target.double().cpu().numpy()
        want = A.weights(q.double().cpu().numpy(), cache.k_np, cache.table_np, cache.lens_np, lse.double().cpu().numpy(), scale,
                         None if given is None else given.double().cpu().numpy(), before, gs_np, pl_np)
        B.moe_attn_weights(q, cache.k, cache.table, cache.lens, lse, d, given, target, gs, pl, cache.k_scale)
        torch.cuda.synchronize()
        got = target.double().cpu().numpy()
        # the exponent's error over at most Hq / Hkv weights, and the additions' roundings
        tol = (np.expm1(e) + (Hq // Hkv + 64) * U.U_FP32) * (np.abs(want) + 1)
        assert (np.abs(got - want) <= tol).all()
        for r, n in enumerate(lens):
            assert np.array_equal(got[r, :, n:], before[r, :, n:])


def test_weights_of_absent_pages_stay():
    G.say("case: weights, absent pages")
    cache = U.Cache([100, 40], 2, 64, 16, seed=3)
    cache.table_np[0, 2], cache.table_np[1, 0] = -1, cache.nb
    cache.table.copy_(torch.from_numpy(cache.table_np))
    q = U.queries(2, 4, 64)
    _, lse = U.run_decode(cache, q)
    w = torch.rand((2, 2, cache.N), device="cuda")
    want = A.weights(q.double().cpu().numpy(), cache.k_np, cache.table_np, [100, 40], lse.double().cpu().numpy(), 0.125,
                     w.double().cpu().numpy(), np.zeros(w.shape))
    out = torch.zeros_like(w)
    B.moe_attn_weights(q, cache.k, cache.table, cache.lens, lse, cache.dims(4), w, out)
    torch.cuda.synchronize()
    assert np.allclose(out.double().cpu().numpy(), want, rtol=1e-5, atol=1e-6)
    assert torch.equal(out[0, :, 32:48], w[0, :, 32:48])


# ----------------------------------------------------------------------------- evict

EVICT = [
    # lens, Hkv, D, bs, budget, recent, protect, fp8, weights
    ([9, 10, 11, 0, 1], 2, 64, 16, 10, 3, None, False, "random"),
    ([65, 64, 63, 200], 3, 64, 16, 64, 0, [0, 1, 2, 3], False, "ties"),
    ([100, 300, 1000, 5000], 2, 128, 16, 77, 20, [4, 90, 0, 16], False, "random"),
    ([2050, 2049, 2048], 4, 128, 32, 2048, 64, None, False, "random"),
    ([700, 129], 1, 256, 16, 128, 128, None, True, "random"),
    ([700, 129], 2, 64, 64, 1, 0, None, True, "odd"),
    ([3000, 1500], 2, 64, 16, 1000, 7, [5, 5], False, "odd"),
    ([513, 640], 2, 128, 16, 511, 0, None, False, "zero"),
    ([20000], 1, 64, 16, 9000, 100, [3], False, "ties"),
    ([70000], 1, 64, 16, 12345, 100, [3], True, "random"),
    ([500, 480, 512], 2, 64, 16, 448, 5, None, False, "ties"),   # one wave a row, its few moves in the same launch
    ([8192, 8140], 1, 128, 16, 8128, 0, [2, 2], True, "zero"),   # 64 moves at most
    ([8193, 8000], 1, 64, 16, 4096, 9, None, False, "odd"),      # the longest rows that eight keys a lane hold, and over
    ([32768, 20000], 1, 64, 16, 16384, 0, None, False, "random"),
]


@pytest.mark.parametrize("lens,Hkv,D,bs,budget,recent,protect,fp8,kind", EVICT)
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(lens, Hkv, D, bs, budget, recent, protect, fp8, kind, in_place):
    G.say(f"case: evict lens={lens} Hkv={Hkv} D={D} bs={bs} budget={budget} recent={recent} {kind} in_place={in_place}")
    R = len(lens)
    cache = U.Cache(lens, Hkv, D, bs, fp8, seed=budget, pad=64)
    N, rng = cache.N, np.random.default_rng(budget)
    w = rng.exponential(1.0, (R, Hkv, N)).astype(np.float32)
    if kind == "ties":
        w = np.floor(w * 2).astype(np.float32)
    elif kind == "zero":
        w[:] = 0.0
        w[..., ::2] = -0.0
    elif kind == "odd":
        w = np.where(rng.random(w.shape) < 0.3, rng.choice(np.float32([np.nan, np.inf, -np.inf, -1.0, 0.0, -0.0, 1e-42]), w.shape), w)
    gap = 50
    pos = np.stack([np.stack([rng.permutation(N) + gap * (rng.random() < 0.5) for _ in range(Hkv)]) for _ in range(R)]).astype(np.int32)
    seen = np.array([n + gap for n in lens], np.int32)
    src, new, w2, p2 = A.evict(w, pos, lens, seen, budget, recent, protect)
    want = [A.moved(c.float().cpu().numpy(), cache.table_np, src, lens, budget) for c in (cache.k, cache.v)]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    w_d, p_d = dev(w), dev(pos)
    w_out, p_out = (w_d, p_d) if in_place else (dev(w), dev(pos))
    src_d = torch.full((R, Hkv, budget), -9, dtype=torch.int32, device="cuda")
    new_d = torch.empty(R, dtype=torch.int32, device="cuda")
    B.moe_kv_evict(w_d, p_d, cache.lens, dev(seen), cache.table, cache.dims(Hkv), budget, recent, cache.k, cache.v, src_d,
                   new_d, w_out, p_out, protect=None if protect is None else dev(np.array(protect, np.int32)))
    torch.cuda.synchronize()
    assert np.array_equal(src_d.cpu().numpy(), src)
    assert np.array_equal(new_d.cpu().numpy(), new)
    assert np.array_equal(w_out.cpu().numpy().view(np.int32), w2.view(np.int32))
    assert np.array_equal(p_out.cpu().numpy(), p2)
    for got, ref in zip((cache.k, cache.v), want):
        assert np.array_equal(got.float().cpu().numpy(), ref, equal_nan=True)


def test_evict_moves_no_row_of_an_absent_page_and_ignores_extreme_positions():
    G.say("case: evict, absent pages, positions and counts at the ends of int32")
    cache = U.Cache([40], 1, 64, 16, seed=1)
    cache.table_np[0, 0] = -1
    cache.table.copy_(torch.from_numpy(cache.table_np))
    w = np.arange(cache.N, dtype=np.float32)[None, None]
    pos = np.full((1, 1, cache.N), -2 ** 31, np.int32)
    pos[0, 0, 1] = 2 ** 31 - 1
    seen = np.array([-2 ** 31], np.int32)  # seen - recent is below every int32
    before = [c.float().cpu().numpy() for c in (cache.k, cache.v)]
    for recent in (0, 2 ** 31 - 1):
        src, new, w2, p2 = A.evict(w, pos, [40], seen, 20, recent)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        out = dev(np.zeros((1, 1, 20), np.int32)), dev(new.astype(np.int32)), dev(w), dev(pos)
        B.moe_kv_evict(dev(w), dev(pos), cache.lens, dev(seen), cache.table, cache.dims(1), 20, recent, cache.k, cache.v, *out)
        torch.cuda.synchronize()
        assert np.array_equal(out[0].cpu().numpy(), src)
        before = [A.moved(c, cache.table_np, src, [40], 20) for c in before]
        for got, ref in zip((cache.k, cache.v), before):
            assert np.array_equal(got.float().cpu().numpy(), ref, equal_nan=True)
