"""A decode worker's steps on one layer: attention over the paged KV cache, then the
MoE layer, for a batch whose requests share their domain's prompt.

    python examples/decode_step.py [--requests 64] [--prefix 2048] [--own 256] [--budget 2304] [--steps 20]
                                   [--fp8 | --int8] [--norm]

Each step, all on one stream and without a host synchronisation:

  1. project the batch's hidden states to queries, keys and values
  2. moe_kv_append    rotate them by their positions, store keys and values
                      (--norm: moe_kv_append_norm, queries and keys normed first;
                      --int8: moe_kv_append_int8, into 8-bit integers)
  3. moe_attn_decode  attend; the shared prompt is read once for its group
  4. project back, and run the MoE layer (moe_layer)
  5. moe_attn_weights add to each cached token's accumulated attention weight
  6. moe_kv_evict     requests over their budget lose their lightest tokens

A cache of 8-bit integers has a scale for each page and does without 5 and 6, so the
budget has to hold every step's token, and does where none is given.

Random weights and hidden states; the projections are torch's, everything else is
the library's.
"""
from __future__ import annotations

import argparse
import os
import sys
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_00466_amd import binding as B  # noqa: E402
from paper_2607_00466_amd import synth  # noqa: E402

BLOCK = 16
RECENT = 32  # tokens that are never evicted


@dataclass
class Heads:
    Hq: int
    Hkv: int
    D: int


def check_sizes(groups, prefix, own, budget, steps, recent=RECENT, fp8=False, int8=False):
    if prefix % BLOCK or budget < prefix + recent:
        raise ValueError("the prefix is whole pages, and the budget holds it and the recent tokens")
    if steps < 1 or own < 0 or groups < 1:
        raise ValueError("a worker has a step to make, a group and no fewer than 0 tokens of its own a request")
    if int8 and (fp8 or budget < prefix + own + steps):
        raise ValueError("a cache of 8-bit integers is none of fp8, and nothing is evicted from it: the budget holds every token")


class Worker:
    """One layer's weights, and the batch's cache: `groups` equal groups of requests,
    each behind `prefix` shared tokens and with `own` tokens of its own, with room
    for `steps` steps."""

    def __init__(self, shape: synth.LayerShape, heads: Heads, R: int, groups: int, prefix: int, own: int, budget: int,
                 steps: int, recent: int = RECENT, fp8: bool = False, int8: bool = False, norm: bool = False, seed: int = 0):
        check_sizes(groups, prefix, own, budget, steps, recent, fp8, int8)
        self.left = steps
        self.shape, self.heads, self.budget, self.recent = shape, heads, budget, recent
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s, std=1.0: torch.empty(s, device="cuda").normal_(0, std, generator=gen)  # noqa: E731
        i32 = dict(dtype=torch.int32, device="cuda")
        Hq, Hkv, D, H = heads.Hq, heads.Hkv, heads.D, shape.H
        # weights
        self.w_qkv = normal(H, (Hq + 2 * Hkv) * D, std=H ** -0.5).bfloat16()
        self.w_out = normal(Hq * D, H, std=(Hq * D) ** -0.5).bfloat16()
        self.w_gate = torch.from_numpy(synth.gate_weights(shape, seed)).cuda()
        self.experts = B.pack_expert_weights(*synth.expert_weights(shape, seed, device="cuda"))
        angle = torch.arange(prefix + own + steps + 1, device="cuda", dtype=torch.float64)[:, None] * \
            1e6 ** (-torch.arange(D // 2, device="cuda", dtype=torch.float64) * 2 / D)
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        self.pair_axis = torch.zeros(D // 2, **i32)  # text: one position axis
        self.q_norm, self.k_norm = (1 + normal(D, std=0.1) if norm else None for _ in "qk")
        # pages: each group's shared ones, then each request's own (room for every step, or for the budget and one more)
        most = min(prefix + own + steps, max(budget, prefix + own) + 1)
        shared, private = prefix // BLOCK, -(-(most - prefix) // BLOCK)
        nb = groups * shared + R * private
        ids = torch.randperm(nb, device="cuda", generator=gen).to(torch.int32)
        start = [g * R // groups for g in range(groups + 1)]
        table = torch.empty((R, shared + private), **i32)
        table[:, shared:] = ids[groups * shared:].view(R, private)
        for g in range(groups):
            table[start[g]:start[g + 1], :shared] = ids[g * shared:(g + 1) * shared]
        self.table = table
        self.group_start = torch.tensor(start, **i32)
        self.prefix_len = torch.full((groups,), prefix, **i32)
        self.protect = torch.full((R,), prefix, **i32)
        kv = torch.int8 if int8 else torch.float8_e4m3fn if fp8 else torch.bfloat16
        self.d = B.attn_dims(R, Hq, Hkv, D, BLOCK, table.shape[1], nb, kv)
        self.k_cache, self.v_cache = (torch.zeros((nb, Hkv, BLOCK, D), device="cuda").to(kv) for _ in "kv")
        self.k_scale = self.v_scale = torch.full((Hkv,), 1 / 64, device="cuda") if fp8 else None
        if int8:
            self.k_scale, self.v_scale = (torch.zeros((nb, Hkv), device="cuda") for _ in "kv")
        self.int8 = int8
        self.N = table.shape[1] * BLOCK
        # per slot: the token's position, and the attention it has received
        self.pos = torch.full((R, Hkv, self.N), -1, **i32)
        self.weights = torch.zeros((R, Hkv, self.N), device="cuda")
        self.lens = torch.zeros(R, **i32)
        self.seen = torch.zeros(R, **i32)
        # buffers of a step, allocated once
        self.ws = B.attn_workspace(self.d)
        self.q = torch.empty((R, Hq, D), dtype=torch.bfloat16, device="cuda")
        self.out, self.lse = torch.empty_like(self.q), torch.empty((R, Hq), device="cuda")
        self.src, self.new_lens = torch.empty((R, Hkv, budget), **i32), torch.empty(R, **i32)
        self.moe_d = B.dims(R, H, shape.E, shape.K, shape.I)
        self.moe = B.LayerBuffers.allocate(self.moe_d)
        self.rows = torch.arange(R, device="cuda")
        self.each = torch.arange(R + 1, **i32)  # a token of each request
        self._prompt(normal, start, prefix, own)

    def _append(self, x, positions, rows, index, q_out):
        """Project x [T, H] and store its keys and values at slots `index` of requests
        `rows` (one, or one a token); queries into q_out where wanted."""
        h, T = self.heads, x.shape[0]
        if T == 0:
            return
        qkv = (x.bfloat16() @ self.w_qkv).view(T, h.Hq + 2 * h.Hkv, h.D)
        q = qkv[:, :h.Hq] if q_out is not None else None
        new = (q, qkv[:, h.Hq:h.Hq + h.Hkv], qkv[:, h.Hq + h.Hkv:], positions[None], self.pair_axis, self.cos, self.sin)
        if self.int8:
            one = isinstance(rows, int)  # a run of tokens of one request, or a token of each
            table = self.table[rows:rows + 1] if one else self.table
            d = B.attn_dims(len(table), h.Hq, h.Hkv, h.D, BLOCK, self.d.max_blocks, self.d.num_blocks, torch.int8)
            start = torch.tensor([0, T], dtype=torch.int32, device="cuda") if one else self.each
            B.moe_kv_append_int8(*new, start, table, index[:1].int() if one else index.int(), d, q_out, self.k_cache, self.v_cache,
                                 self.k_scale, self.v_scale, self.q_norm, self.k_norm)
            return
        after = (self._slots(rows, index), self.d, q_out, self.k_cache, self.v_cache)
        if self.q_norm is not None:
            B.moe_kv_append_norm(*new, *after, self.q_norm, self.k_norm, k_scale=self.k_scale, v_scale=self.v_scale)
        else:
            B.moe_kv_append(*new, *after, self.k_scale, self.v_scale)

    def _slots(self, rows, index):
        """Cache slots of slot `index` of requests `rows`."""
        return self.table[rows, index // BLOCK] * BLOCK + (index % BLOCK).to(torch.int32)

    def _prompt(self, normal, start, prefix, own):
        """The shared prompts, once a group, then each request's own part."""
        H = self.shape.H
        for g in range(len(start) - 1):
            at = torch.arange(prefix, device="cuda")
            if prefix:
                self._append(normal(prefix, H), at.int(), start[g], at, None)
        for r in range(self.d.R):
            at = torch.arange(prefix, prefix + own, device="cuda")
            self._append(normal(own, H), at.int(), r, at, None)
        self.pos[:, :, :prefix + own] = torch.arange(prefix + own, device="cuda", dtype=torch.int32)
        self.lens.fill_(prefix + own)
        self.seen.fill_(prefix + own)

    def attend(self, x):
        """Steps 1 to 3: the new tokens into the cache, and their attention."""
        if self.left <= 0:
            raise RuntimeError("the cache and the rotation tables have room for no further step")
        self.left -= 1
        at = self.lens.long()
        self._append(x, self.seen, self.rows, at, self.q)
        self.pos[self.rows, :, at] = self.seen[:, None]
        self.lens += 1
        self.seen += 1
        B.moe_attn_decode(self.q, self.k_cache, self.v_cache, self.table, self.lens, self.d, self.out, self.lse, self.ws,
                          self.group_start, self.prefix_len, self.k_scale, self.v_scale)
        return self.out

    def evict(self):
        """Steps 5 and 6."""
        if self.int8:
            return
        B.moe_attn_weights(self.q, self.k_cache, self.table, self.lens, self.lse, self.d, self.weights, self.weights,
                           self.group_start, self.prefix_len, self.k_scale)
        B.moe_kv_evict(self.weights, self.pos, self.lens, self.seen, self.table, self.d, self.budget, self.recent,
                       self.k_cache, self.v_cache, self.src, self.new_lens, self.weights, self.pos, protect=self.protect)
        self.lens.copy_(self.new_lens)

    def step(self, x):
        """One decode step: hidden states x [R, H] fp32 in, the layer's output."""
        x = x + (self.attend(x).view(x.shape[0], -1) @ self.w_out).float()
        x = x + B.moe_layer(x, self.w_gate, *self.experts, self.moe_d, self.moe)
        self.evict()
        return x


def arguments(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--shape", default="qwen3_30b_a3b", choices=sorted(synth.SHAPES))
    p.add_argument("--heads", type=int, nargs=3, default=(32, 4, 128), metavar=("HQ", "HKV", "D"))
    p.add_argument("--requests", type=int, default=64)
    p.add_argument("--groups", type=int, default=1)
    p.add_argument("--prefix", type=int, default=2048)
    p.add_argument("--own", type=int, default=256)
    p.add_argument("--budget", type=int, help="default 2304; with --int8 every token of the run")
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--fp8", action="store_true")
    p.add_argument("--int8", action="store_true")
    p.add_argument("--norm", action="store_true")
    a = p.parse_args(argv)
    if a.budget is None:
        a.budget = a.prefix + max(a.own + a.steps, RECENT) if a.int8 else 2304
    return a


def main(argv=None):
    a = arguments(argv)
    w = Worker(synth.SHAPES[a.shape], Heads(*a.heads), a.requests, a.groups, a.prefix, a.own, a.budget, a.steps, fp8=a.fp8,
               int8=a.int8, norm=a.norm)
    x = torch.randn((a.requests, w.shape.H), device="cuda")
    y = w.step(x)
    torch.cuda.synchronize()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in "be")
    begin.record()
    for _ in range(a.steps - 1):
        y = w.step(x)
    end.record()
    torch.cuda.synchronize()
    took = f"{begin.elapsed_time(end) / (a.steps - 1) * 1e3:.1f} us a step" if a.steps > 1 else "one step, not timed"
    print(f"{a.requests} requests, {a.groups} x {a.prefix} shared + {a.own} own tokens: {took}; "
          f"union {int(w.moe.union_size.item())}, {int(w.lens[0].item())} tokens cached of {int(w.seen[0].item())} seen, "
          f"output {float(y.abs().mean()):.3f} mean |y|")
    return y


if __name__ == "__main__":
    main()
