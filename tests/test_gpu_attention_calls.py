"""How the attention calls may be made: on other streams, in graphs, with block strides,
with the largest plan."""
import numpy as np
import pytest
import torch

from oracle import attention as A
from paper_2607_00466_amd import binding as B
from tests import attention_util as U
from tests import gpu_util as G

pytestmark = pytest.mark.gpu


class Step:
    """The calls of a step on fixed buffers: `reset` brings inputs and outputs back."""

    def __init__(self, R=6, Hq=8, Hkv=2, D=64, bs=16, prefix=64, budget=130):
        self.R, self.Hq, self.Hkv, self.D, self.budget = R, Hq, Hkv, D, budget
        lens = [prefix + 40 + 23 * i for i in range(R)]
        self.shared = ((0, R, prefix),)
        self.cache = c = U.Cache(lens, Hkv, D, bs, seed=11, shared=self.shared, max_blocks=-(-(max(lens) + 8) // bs))
        # the group's members have the prefix' pages in their rows
        c.table_np[:, :prefix // bs] = c.table_np[0, :prefix // bs]
        c.table.copy_(torch.from_numpy(c.table_np))
        self.d = c.dims(Hq)
        self.gs, self.pl, _, _ = U.groups_of(self.shared, R)
        g = torch.Generator(device="cuda").manual_seed(5)
        i32 = dict(dtype=torch.int32, device="cuda")
        angle = torch.arange(400, device="cuda", dtype=torch.float64)[:, None] * 0.7 ** torch.arange(D // 2, device="cuda")
        self.cos, self.sin, self.axis = angle.cos().float(), angle.sin().float(), torch.zeros(D // 2, **i32)
        self.rows = torch.randn((R, Hq + 2 * Hkv, D), device="cuda", generator=g)
        at = c.lens.long() - 1  # the last cached slot is the new token's
        self.slots = (c.table[torch.arange(R, device="cuda"), at // bs].long() * bs + at % bs).to(torch.int32)
        self.positions = (c.lens - 1)[None].contiguous()
        self.q = torch.empty((R, Hq, D), dtype=torch.bfloat16, device="cuda")
        self.out, self.lse = torch.empty_like(self.q), torch.empty((R, Hq), device="cuda")
        self.ws = B.attn_workspace(self.d)
        self.weights = torch.empty((R, Hkv, c.N), device="cuda")
        self.pos = torch.empty((R, Hkv, c.N), **i32)
        self.protect = torch.full((R,), prefix, **i32)
        self.seen = c.lens.clone()
        self.src, self.new_lens = torch.empty((R, Hkv, budget), **i32), torch.empty(R, **i32)
        self.start = [t.clone() for t in (c.k, c.v)]
        self.w0 = torch.rand(self.weights.shape, device="cuda", generator=g)
        self.outputs = (self.q, c.k, c.v, self.out, self.lse, self.weights, self.pos, self.src, self.new_lens)

    def reset(self):
        self.cache.k.copy_(self.start[0]), self.cache.v.copy_(self.start[1])
        self.weights.copy_(self.w0)
        self.pos.copy_(torch.arange(self.cache.N, device="cuda").expand_as(self.pos))
        for t in (self.q, self.out, self.lse):
            t.fill_(float("nan"))
        self.src.fill_(-9), self.new_lens.fill_(-9)

    def run(self, stream=None):
        c, h = self.cache, self.Hq
        B.moe_kv_append(self.rows[:, :h], self.rows[:, h:h + self.Hkv], self.rows[:, h + self.Hkv:], self.positions, self.axis,
                        self.cos, self.sin, self.slots, self.d, self.q, c.k, c.v, stream=stream)
        B.moe_attn_decode(self.q, c.k, c.v, c.table, c.lens, self.d, self.out, self.lse, self.ws, self.gs, self.pl, stream=stream)
        B.moe_attn_weights(self.q, c.k, c.table, c.lens, self.lse, self.d, self.weights, self.weights, self.gs, self.pl,
                           stream=stream)
        B.moe_kv_evict(self.weights, self.pos, c.lens, self.seen, c.table, self.d, self.budget, 4, c.k, c.v, self.src,
                       self.new_lens, self.weights, self.pos, protect=self.protect, stream=stream)

    def taken(self):
        return [t.clone() for t in self.outputs]


def _same(a, b):
    # (bits: pages that hold nothing are NaN)
    return all(torch.equal(x.view(torch.int16) if x.dtype is torch.bfloat16 else x, y.view(torch.int16) if y.dtype is torch.bfloat16 else y)
               for x, y in zip(a, b))


def test_every_call_on_a_side_stream():
    G.say("case: append, decode, weights and evict on a side stream, given and current")
    s = Step()
    s.reset()
    s.run()
    want = s.taken()
    assert (want[-1].cpu().numpy() == np.minimum(s.cache.lens_np, s.budget)).all()
    assert not want[3].isnan().any()
    side = torch.cuda.Stream()
    for given in (True, False):
        s.reset()
        side.wait_stream(torch.cuda.current_stream())  # after what the reset wrote
        if given:
            s.run(stream=side)
        else:
            with torch.cuda.stream(side):
                s.run()
        torch.cuda.current_stream().wait_stream(side)
        assert _same(s.taken(), want)


def test_every_call_in_a_graph():
    G.say("case: append, decode, weights and evict in one graph, lengths and prefixes changing between replays")
    s = Step()
    s.reset()
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    lens = s.cache.lens.clone()
    for step in range(4):
        s.cache.lens.copy_((lens - 9 * step).clamp_min(0))
        s.seen.copy_(s.cache.lens)
        s.pl.fill_(64 - 16 * step)
        s.reset()
        graph.replay()
        got = s.taken()
        torch.cuda.synchronize()
        s.reset()
        s.run()
        assert _same(got, s.taken())


@pytest.mark.parametrize("D,fp8,Hq,Hkv", [(128, False, 16, 2), (64, True, 8, 2), (256, False, 24, 1)])
def test_weights_over_pages_with_a_stride(D, fp8, Hq, Hkv):
    G.say(f"case: weights over pages with a block stride, D={D} fp8={fp8} heads {Hq}/{Hkv}")
    lens, shared = [150 + 7 * i for i in range(5)], ((0, 3, 144),)
    cache = U.Cache(lens, Hkv, D, 16, fp8, seed=D, shared=shared, pad=96)
    q = U.queries(5, Hq, D)
    _, lse = U.run_decode(cache, q, shared)
    gs, pl, gs_np, pl_np = U.groups_of(shared, 5)
    out = torch.full((5, Hkv, cache.N), -2.0, device="cuda")
    want = A.weights(q.double().cpu().numpy(), cache.k_np, cache.table_np, cache.lens_np, lse.double().cpu().numpy(), D ** -0.5,
                     None, out.double().cpu().numpy(), gs_np, pl_np)
    B.moe_attn_weights(q, cache.k, cache.table, cache.lens, lse, cache.dims(Hq), None, out, gs, pl, cache.k_scale)
    torch.cuda.synchronize()
    tol = (np.expm1(U.score_bound(q, cache, D ** -0.5)) + (Hq // Hkv + 64) * U.U_FP32) * (np.abs(want) + 1)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("D,fp8", [(256, False), (64, True)])
def test_weights_of_most_requests_and_groups(D, fp8):
    G.say(f"case: weights of 1024 requests in 512 groups of two, D={D}: the largest plan")
    rng = np.random.default_rng(D)
    lens, shared = [int(x) for x in rng.integers(0, 40, 1024)], []
    for s in range(0, 1024, 2):
        n = 16 * int(rng.integers(0, 3))
        shared.append((s, s + 2, n))
        lens[s] += n
        lens[s + 1] += n
    cache = U.Cache(lens, 1, D, 16, fp8, seed=D, shared=shared)
    q = U.queries(1024, 2, D)
    first, lse = U.run_decode(cache, q, shared)
    gs, pl, gs_np, pl_np = U.groups_of(shared, 1024)
    # as many groups as a call takes: the others are empty
    gs = torch.cat([gs, torch.full((1024 - pl.numel(),), 1024, dtype=torch.int32, device="cuda")])
    pl = torch.cat([pl, torch.zeros(1024 - pl.numel(), dtype=torch.int32, device="cuda")])
    again, lse2 = torch.empty_like(first), torch.empty_like(lse)
    d = cache.dims(2)
    B.moe_attn_decode(q, cache.k, cache.v, cache.table, cache.lens, d, again, lse2, B.attn_workspace(d), gs, pl, cache.k_scale,
                      cache.v_scale)
    assert torch.equal(again, first) and torch.equal(lse2, lse)
    out = torch.full((1024, 1, cache.N), -2.0, device="cuda")
    want = A.weights(q.double().cpu().numpy(), cache.k_np, cache.table_np, cache.lens_np, lse.double().cpu().numpy(), D ** -0.5,
                     None, out.double().cpu().numpy(), gs_np, pl_np)
    B.moe_attn_weights(q, cache.k, cache.table, cache.lens, lse, cache.dims(2), None, out, gs, pl, cache.k_scale)
    torch.cuda.synchronize()
    tol = (np.expm1(U.score_bound(q, cache, D ** -0.5)) + (2 + 64) * U.U_FP32) * (np.abs(want) + 1)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
