"""The int8 cache's calls as a worker makes them: prompts, steps, forked requests that go
on apart, requests that end and pages that move together; in two layers, every step's
attention against the oracle on what the cache holds, and the caches bit for bit.  And
the decode-step example with its norms and its cache of 8-bit integers."""
import numpy as np
import pytest
import torch

from examples import decode_step as E
from oracle import attention as A
from oracle import kv_cache as K
from paper_2607_00466_amd import binding as B
from paper_2607_00466_amd import synth
from tests import attention_util as U
from tests.kv_cache_util import Rows, dev, i32

pytestmark = pytest.mark.gpu

LAYERS, NB, HQ, HKV, BS, D, ROWS, WIDTH = 2, 40, 8, 2, 16, 128, 6, 6


class Worker:
    """Two layers' caches, tables and lengths, on the device and as the oracle has them;
    pages are handed out on the host."""

    def __init__(self):
        rng = np.random.default_rng(0)
        shape = (LAYERS, NB, HKV, BS, D)
        self.np = [rng.integers(-127, 128, shape).astype(np.int8) for _ in "kv"] + \
            [np.full(shape[:3], np.nan, np.float32) for _ in "kv"]
        self.k, self.v, self.ks, self.vs = (dev(x) for x in self.np)
        self.table, self.lens = np.full((ROWS, WIDTH), -1, np.int32), np.zeros(ROWS, np.int32)
        self.free = list(rng.permutation(NB))
        self.d = B.attn_dims(ROWS, HQ, HKV, D, BS, WIDTH, NB, torch.int8)
        self.ws, self.seed = B.attn_workspace(self.d), 0

    def append(self, new):
        """new[r] tokens to each request, in both layers."""
        for r, n in enumerate(new):
            for i in range(-(-int(self.lens[r]) // BS), -(-int(self.lens[r] + n) // BS)):
                self.table[r, i] = self.free.pop()
        start = np.concatenate([[0], np.cumsum(new)])
        T = int(start[-1])
        for layer in range(LAYERS):
            self.seed += 1
            r = Rows(T, HQ, HKV, D, 64, fp32=False, seed=self.seed)
            B.moe_kv_append_int8(r.q, r.k, r.v, r.positions, r.axis, r.cos, r.sin, i32(start), i32(self.table), i32(self.lens),
                                 self.d, r.q_out, self.k[layer], self.v[layer], self.ks[layer], self.vs[layer], r.q_norm, r.k_norm)
            for codes, scale, x in ((0, 2, r.expected("k")), (1, 3, r.numpy("v"))):
                self.np[codes][layer], self.np[scale][layer] = K.append_int8(x, start, self.table, self.lens, self.np[codes][layer],
                                                                             self.np[scale][layer])
            self.q = r.q_out
        self.lens = self.lens + np.asarray(new, np.int32)
        self.check()

    def check(self):
        torch.cuda.synchronize()
        for got, want in zip((self.k, self.v, self.ks, self.vs), self.np):
            np.testing.assert_array_equal(got.cpu().numpy(), want)

    def step(self):
        live = self.lens > 0
        self.append(live.astype(int))
        q = torch.zeros((ROWS, HQ, D), dtype=torch.bfloat16, device="cuda")
        q[torch.from_numpy(live).cuda()] = self.q * 0.1
        out, lse = torch.empty_like(q), torch.empty((ROWS, HQ), device="cuda")
        layer = LAYERS - 1
        B.moe_attn_decode(q, self.k[layer], self.v[layer], i32(self.table), i32(self.lens), self.d, out, lse, self.ws,
                          k_scale=self.ks[layer], v_scale=self.vs[layer])

        class View:
            pass

        view = View()
        view.D = D
        view.k_np, view.v_np = (self.np[c][layer] * self.np[c + 2][layer].astype(np.float64)[:, :, None, None] for c in range(2))
        ref = A.decode(q.double().cpu().numpy(), view.k_np, view.v_np, self.table, self.lens, D ** -0.5)
        U.check_decode(out, lse, q, view, D ** -0.5, ref)

    def fork(self, parent, child):
        page = [self.free.pop() for _ in parent]
        t, n = i32(self.table), i32(self.lens)
        B.moe_kv_fork(i32(parent), i32(child), i32(page), t, n, self.d, self.k, self.v, self.ks, self.vs)
        self.table, self.lens, caches, scales = K.fork(parent, child, page, self.table, self.lens, self.np[:2], self.np[2:])
        self.np = caches + scales
        assert np.array_equal(t.cpu().numpy(), self.table) and np.array_equal(n.cpu().numpy(), self.lens)
        self.check()

    def end(self, rows):
        for r in rows:
            self.table[r], self.lens[r] = -1, 0

    def compact(self):
        held = sorted({int(b) for b in self.table.flat if b >= 0})
        remap = np.full(NB, -1, np.int32)
        remap[held] = held
        for b, to in zip([b for b in held if b >= len(held)], [b for b in range(len(held)) if remap[b] < 0]):
            remap[b] = to
        t = i32(self.table)
        B.moe_kv_compact(i32(remap), t, t, self.d, self.k, self.v, self.ks, self.vs)
        self.table, caches, scales = K.compact(remap, self.table, self.np[:2], self.np[2:])
        self.np = caches + scales
        assert np.array_equal(t.cpu().numpy(), self.table) and self.table.max() < len(held)
        self.free = list(range(len(held), NB))
        self.check()


def test_a_workers_life():
    w = Worker()
    w.append([21, 16, 5, 0, 0, 0])   # prompts
    w.step()
    w.fork([0, 0, 2], [3, 4, 5])     # three more answers: full pages are shared, the last ones copied
    for _ in range(12):              # each goes on in pages of its own
        w.step()
    w.end([0, 1])
    w.compact()
    for _ in range(6):
        w.step()
    w.fork([4], [0])
    w.end([4, 2])
    w.compact()
    w.append([3, 17, 0, 1, 0, 18])   # a new prompt beside requests that go on
    w.step()


@pytest.mark.parametrize("int8,fp8", [(True, False), (False, True), (False, False)])
def test_example_steps_match_the_oracle(int8, fp8):
    w = E.Worker(synth.SHAPES["tiny"], E.Heads(8, 2, 64), R=6, groups=2, prefix=32, own=20, budget=60, steps=8, recent=4, fp8=fp8,
                 int8=int8, norm=True)
    table, gs, pl = w.table.cpu().numpy(), w.group_start.tolist(), w.prefix_len.tolist()
    x = torch.randn((6, w.shape.H), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    for step in range(8):
        out = w.attend(x)
        torch.cuda.synchronize()

        class View:
            pass

        view = View()
        view.D = 64
        scales = [1.0 if s is None else s.double().cpu().numpy().reshape(-1, 2)[:, :, None, None] for s in (w.k_scale, w.v_scale)]
        view.k_np, view.v_np = (c.cpu().double().numpy() * s for c, s in zip((w.k_cache, w.v_cache), scales))
        assert w.lens.tolist() == [53 + step] * 6
        # queries and keys are normed: each head's mean square is about its weights'
        assert 0.9 < float(w.q.float().square().mean(-1).sqrt().mean()) < 1.1
        ref = A.decode(w.q.double().cpu().numpy(), view.k_np, view.v_np, table, w.lens.cpu().numpy(), 64 ** -0.5, gs, pl)
        U.check_decode(out, w.lse, w.q, view, 64 ** -0.5, ref)
        w.evict()


def test_example_runs_with_8_bit_integers():
    y = E.main(["--shape", "tiny", "--heads", "4", "2", "64", "--requests", "5", "--prefix", "32", "--own", "9", "--budget", "64",
                "--steps", "3", "--int8", "--norm"])
    assert y.shape == (5, synth.SHAPES["tiny"].H) and bool(torch.isfinite(y).all())
