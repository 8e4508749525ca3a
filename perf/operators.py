"""The attention half of a decode step over the paged KV cache: what is measured of its operators.

Four operators, as a decode worker runs them around its MoE layers:

  append   rotary positions (one axis or several) of the new tokens' queries and keys, and
           the write of keys and values into the cache's pages
  attend   one query token a request against its cached tokens, prefixes that requests share
           read once for the group
  weigh    each cached token's attention weight, added to what it has accumulated
  evict    the tokens of largest accumulated weight stay, the cache is compacted in place

``run`` computes them by elementary torch operations, or, where ``own`` is true, by the
library's entry points.  Shapes are those of the decode layers this repository names
(batches of 1 to 256 requests; 32 query heads over 4 of 128, 64 over 8 of 64, block size 16)
and generic ones near them.
"""
import functools
import math
import random

import numpy as np
import torch

own = False

BF16, FP8 = torch.bfloat16, torch.float8_e4m3fn
FP8_MAX = 448.0


# ----------------------------------------------------------------------------- cases

def _append(name, T, Hq, Hkv, D, rot, axes=1, interleaved=False, fp8=False, fp32=False, bs=16):
    """T new tokens: queries and keys rotated, keys and values written to their pages."""
    return dict(name=name, op="append", T=T, Hq=Hq, Hkv=Hkv, D=D, rot=rot, axes=axes,
                interleaved=interleaved, fp8=fp8, fp32=fp32, bs=bs)


def _attn(name, op, R, Hq, Hkv, D, lo, hi, groups=0, prefix=0, fp8=False, window=0, sinks=False, bs=16):
    """R requests with lo to hi cached tokens of their own each, after a prefix of
    ``prefix`` tokens that each of ``groups`` equal groups shares."""
    return dict(name=name, op=op, R=R, Hq=Hq, Hkv=Hkv, D=D, lo=lo, hi=hi, groups=groups,
                prefix=prefix, fp8=fp8, window=window, sinks=sinks, bs=bs)


def _evict(name, R, Hkv, D, lo, hi, budget, recent, protect=0, fp8=False, bs=16):
    """R requests with lo to hi cached tokens, cut to ``budget``."""
    return dict(name=name, op="evict", R=R, Hkv=Hkv, D=D, lo=lo, hi=hi, budget=budget,
                recent=recent, protect=protect, fp8=fp8, bs=bs)


def listed():
    return [
        # the new token of each request of a decode batch: latency counts
        _append("append 64 new tokens", 64, 32, 4, 128, 128),
        # a prompt with images: three position axes, activations in fp32
        _append("append 4096 in three axes", 4096, 32, 4, 128, 128, axes=3, fp32=True),
        # an odd prompt into an fp8 cache, half of each head rotated, pairs side by side
        _append("append 1001 to an fp8 cache", 1001, 64, 8, 64, 32, interleaved=True, fp8=True),
        # few requests, short contexts: latency counts
        _attn("attend 8 of up to 512", "attend", 8, 32, 4, 128, 1, 512),
        # an ordinary batch of mixed lengths, nothing shared
        _attn("attend 128 of up to 8000", "attend", 128, 32, 4, 128, 17, 8000),
        # two requests with very long contexts: the work of a row split over the chip
        _attn("attend 2 near 131000 in fp8", "attend", 2, 32, 4, 128, 129999, 131071, fp8=True),
        # a domain's batch behind one long system prompt
        _attn("attend 64 behind 8192", "attend", 64, 32, 4, 128, 33, 700, groups=1, prefix=8192),
        # a large batch of several domains, 64-wide heads with sink logits, fp8
        _attn("attend 256 behind 8 x 2048", "attend", 256, 64, 8, 64, 1, 1500, groups=8,
              prefix=2048, fp8=True, sinks=True),
        # the weights of an ordinary batch, and of a batch behind a shared prompt
        _attn("weigh 64 of up to 4000", "weigh", 64, 32, 4, 128, 17, 4000),
        _attn("weigh 64 behind 8192", "weigh", 64, 32, 4, 128, 33, 700, groups=1, prefix=8192),
        # a batch whose caches are cut to half, at most
        _evict("evict 64 to 2048", 64, 4, 128, 2000, 4096, 2048, 64, protect=4),
        # every step of a batch at its budget: one token out, one in
        _evict("evict one token of 256", 256, 4, 128, 1025, 1025, 1024, 32, protect=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    Hq, Hkv, D = rng.choice([(32, 4, 128), (64, 8, 64), (32, 8, 128), (16, 16, 64), (20, 4, 128), (16, 2, 256)])
    bs = rng.choice([16, 16, 32, 64])
    fp8 = rng.random() < 0.4
    op = rng.choice(["append", "attend", "attend", "weigh", "evict"])
    if op == "append":
        rot = rng.choice([D, D, D // 2])
        c = _append("", _log(rng, 1, 4096), Hq, Hkv, min(D, 128), min(rot, 128), axes=rng.choice([1, 1, 3]),
                    interleaved=rng.random() < 0.3, fp8=fp8, fp32=rng.random() < 0.4, bs=bs)
    elif op == "evict":
        budget = _log(rng, 64, 2048)
        R = _log(rng, 1, 256)
        hi = min(max(budget + 1, _log(rng, budget, 8 * budget)), max(budget + 1, 200000 // R))
        c = _evict("", R, min(Hkv, 4), min(D, 128), max(1, hi // rng.choice([1, 2, 8])), hi, budget,
                   rng.choice([0, 16, budget // 4]), protect=rng.choice([0, 4]), fp8=fp8, bs=bs)
    else:
        shared = rng.random() < 0.5
        R = _log(rng, 2 if shared else 1, 256)
        D = min(D, 128) if R > 64 else D
        groups = rng.choice([1, 1, max(1, R // 16), max(1, R // 3)]) if shared else 0
        # no more products and no more cached bytes than the largest of the listed
        longest = min(8192, 2500000000 // (R * Hq * D))
        prefix = bs * max(1, _log(rng, min(64, longest), longest) // bs) if shared else 0
        rows = (250000000 if shared else 500000000) // (2 * Hkv * D * (1 if fp8 else 2))
        hi = _log(rng, 1, min(131000, max(64, rows // R)))
        plain = not shared and rng.random() < 0.25
        c = _attn("", op, R, Hq, Hkv, D, max(1, hi // rng.choice([1, 4, 64])), hi, groups, prefix,
                  fp8=fp8, window=_log(rng, 16, 1024) if plain and op == "attend" else 0,
                  sinks=rng.random() < 0.3 and op == "attend", bs=bs)
    del c["name"]
    return c


def _lens(case):
    """The requests' private lengths: a fixed draw for the case, its ends among them."""
    r = random.Random("%(R)d %(lo)d %(hi)d" % case)
    lens = [r.randint(case["lo"], case["hi"]) for _ in range(case["R"])]
    lens[-1] = case["hi"]
    return lens


def _bounds(case):
    """The groups' first requests, and R."""
    return [g * case["R"] // case["groups"] for g in range(case["groups"] + 1)]


def work(case):
    c = case
    e = 1 if c.get("fp8") else 2
    if c["op"] == "append":
        rows = c["T"] * c["D"]
        n_in = (c["Hq"] + 2 * c["Hkv"]) * rows * (4 if c["fp32"] else 2)
        return {"bytes": n_in + c["Hq"] * rows * 2 + 2 * c["Hkv"] * rows * e + 4 * c["T"] * (1 + c["axes"] + c["rot"]),
                "flops": 3 * c["T"] * (c["Hq"] + c["Hkv"]) * c["rot"]}
    lens = _lens(c)
    if c["op"] == "evict":
        # the expected share of the kept tokens that lie past the budget, where weights are drawn alike
        cut = [n for n in lens if n > c["budget"]]
        moved = sum(c["budget"] * (n - c["budget"]) / n for n in cut) * c["Hkv"]
        return {"bytes": 4 * moved * c["D"] * e + 16 * sum(lens) * c["Hkv"], "flops": 0}
    kept = [min(n, c["window"]) if c["window"] else n for n in lens]
    distinct = sum(kept) + c["groups"] * c["prefix"]
    seen = sum(kept) + c["R"] * c["prefix"]
    row = c["Hkv"] * c["D"]
    if c["op"] == "attend":
        return {"bytes": distinct * 2 * row * e + c["R"] * c["Hq"] * (4 * c["D"] + 4), "flops": 4 * seen * c["Hq"] * c["D"]}
    return {"bytes": distinct * row * e + seen * c["Hkv"] * 8 + c["R"] * c["Hq"] * (2 * c["D"] + 4),
            "flops": 2 * seen * c["Hq"] * c["D"]}


# ----------------------------------------------------------------------------- inputs

def _pages(shape, gen, fp8, amp=1.0):
    x = torch.empty(shape, dtype=BF16, device="cuda").normal_(0, amp, generator=gen)
    return x.to(FP8) if fp8 else x


def _scales(Hkv, fp8, gen):
    if not fp8:
        return None
    return 0.5 + torch.rand(Hkv, device="cuda", generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = random.Random(seed)
    return {"append": _prepare_append, "evict": _prepare_evict}.get(case["op"], _prepare_attn)(case, gen, host)


def _prepare_append(case, gen, host):
    T, Hq, Hkv, D, bs, rot = (case[k] for k in ("T", "Hq", "Hkv", "D", "bs", "rot"))
    s = dict(case, max_pos=40960)
    # queries, keys and values as one projection leaves them: views of its rows
    qkv = torch.empty((T, Hq + 2 * Hkv, D), device="cuda", dtype=torch.float32 if case["fp32"] else BF16)
    qkv.normal_(generator=gen)
    s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    if case["axes"] == 1:
        # a prompt's positions, or a decode batch's
        if T > 256:
            s["positions"] = torch.arange(T, device="cuda", dtype=torch.int32)[None] + host.randrange(30000)
        else:
            s["positions"] = torch.randint(0, s["max_pos"], (1, T), device="cuda", dtype=torch.int32, generator=gen)
    else:
        # text, an image of side x side patches (its time stands still), text again
        t = torch.arange(T, device="cuda", dtype=torch.int32)
        side = max(1, int(math.sqrt(T / 2)))
        first = T // 4
        i = (t - first).clamp(0, side * side - 1)
        inside = (t >= first) & (t < first + side * side)
        after = torch.where(t < first, t, t - side * side + side)
        s["positions"] = torch.stack([torch.where(inside, first, after), torch.where(inside, first + i // side, after),
                                      torch.where(inside, first + i % side, after)]).to(torch.int32).contiguous()
    # each axis a run of frequencies, the time axis the highest ones
    edges = [a * (rot // 2) // case["axes"] for a in range(1, case["axes"])]
    s["pair_axis"] = torch.tensor([sum(i >= e for e in edges) for i in range(rot // 2)], device="cuda", dtype=torch.int32)
    freq = 1e6 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / rot)
    angle = torch.arange(s["max_pos"], device="cuda", dtype=torch.float64)[:, None] * freq
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    nb = -(-T // bs) + 7
    blocks = torch.randperm(nb, device="cuda", generator=gen)
    i = torch.arange(T, device="cuda")
    s["slots"] = (blocks[i // bs] * bs + i % bs).to(torch.int32)
    s["k_scale"], s["v_scale"] = _scales(Hkv, case["fp8"], gen), _scales(Hkv, case["fp8"], gen)
    shape = (nb, Hkv, bs, D)
    s["k_cache"], s["v_cache"] = (torch.zeros(shape, device="cuda", dtype=BF16).to(FP8 if case["fp8"] else BF16) for _ in "kv")
    s["q_out"] = torch.empty((T, Hq, D), device="cuda", dtype=BF16)
    s["num_blocks"] = nb
    return s


def _tables(case, lens, host):
    """Block tables over scattered pages, shared prefixes on shared pages."""
    bs, prefix = case["bs"], case.get("prefix", 0)
    groups = _bounds(case) if case.get("groups") else []
    own_blocks = [-(-n // bs) for n in lens]
    nb = sum(own_blocks) + len(groups[1:]) * (prefix // bs) + 5
    ids = list(range(nb))
    host.shuffle(ids)
    shared = [[ids.pop() for _ in range(prefix // bs)] for _ in groups[1:]]
    rows = []
    for r, n in enumerate(own_blocks):
        g = next((g for g in range(len(shared)) if groups[g] <= r < groups[g + 1]), None)
        rows.append((shared[g] if g is not None else []) + [ids.pop() for _ in range(n)])
    width = max(len(t) for t in rows)
    table = torch.tensor([t + [-1] * (width - len(t)) for t in rows], dtype=torch.int32, device="cuda")
    return table, nb, width


def _prepare_attn(case, gen, host):
    R, Hq, Hkv, D, bs = (case[k] for k in ("R", "Hq", "Hkv", "D", "bs"))
    s = dict(case)
    lens = _lens(case)
    s["block_table"], s["num_blocks"], s["max_blocks"] = _tables(case, lens, host)
    total = [n + case["prefix"] for n in lens]
    s["longest"] = max(total)
    s["lens"] = torch.tensor(total, dtype=torch.int32, device="cuda")
    s["group_start"] = s["prefix_len"] = None
    if case["groups"]:
        s["group_start"] = torch.tensor(_bounds(case), dtype=torch.int32, device="cuda")
        s["prefix_len"] = torch.full((case["groups"],), case["prefix"], dtype=torch.int32, device="cuda")
    shape = (s["num_blocks"], Hkv, bs, D)
    s["k_cache"] = _pages(shape, gen, case["fp8"])
    s["v_cache"] = _pages(shape, gen, case["fp8"])
    s["k_scale"], s["v_scale"] = _scales(Hkv, case["fp8"], gen), _scales(Hkv, case["fp8"], gen)
    # scores of spread 2: some tokens stand out, as they do in a trained model
    s["q"] = torch.empty((R, Hq, D), dtype=BF16, device="cuda").normal_(0, 2, generator=gen)
    s["sinks"] = torch.empty(Hq, device="cuda").normal_(2, 1, generator=gen) if case["sinks"] else None
    s["out"] = torch.empty((R, Hq, D), dtype=BF16, device="cuda")
    s["lse"] = torch.empty((R, Hq), dtype=torch.float32, device="cuda")
    if case["op"] == "weigh":
        s["lse"] = _plain_softmax(s)[2]
        N = s["max_blocks"] * bs
        seen = torch.arange(N, device="cuda") < s["lens"][:, None, None]
        s["weights"] = torch.empty((R, Hkv, N), device="cuda").exponential_(4.0, generator=gen) * seen
        s["weights_out"] = torch.zeros_like(s["weights"])
    return s


def _prepare_evict(case, gen, host):
    R, Hkv, D, bs, budget = (case[k] for k in ("R", "Hkv", "D", "bs", "budget"))
    s = dict(case)
    lens = _lens(case)
    s["block_table"], s["num_blocks"], s["max_blocks"] = _tables(case, lens, host)
    s["Hq"] = Hkv
    N = s["max_blocks"] * bs
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    n = s["lens"][:, None, None]
    slot = torch.arange(N, device="cuda", dtype=torch.int32)
    # earlier evictions left the tokens in any order, with a gap in their positions
    gap = 1000
    s["seen"] = s["lens"] + gap
    mixed = torch.rand((R, Hkv, N), device="cuda", generator=gen) + 2 * (slot >= n)
    rank = torch.empty((R, Hkv, N), device="cuda", dtype=torch.int32)
    rank.scatter_(2, mixed.argsort(2), slot.expand(R, Hkv, N).contiguous())
    s["pos"] = torch.where(slot < n, torch.where(rank < n // 2, rank, rank + gap), -1).to(torch.int32)
    # accumulated weights: many small, some none at all (equal: the lowest slots stay)
    w = torch.empty((R, Hkv, N), device="cuda").exponential_(1.0, generator=gen) ** 3
    s["weights"] = torch.where((slot < n) & (torch.rand((R, Hkv, N), device="cuda", generator=gen) > 0.05), w, 0.0)
    s["protect_rows"] = torch.full((R,), case["protect"], dtype=torch.int32, device="cuda")
    shape = (s["num_blocks"], Hkv, bs, D)
    s["k_cache"], s["v_cache"] = _pages(shape, gen, case["fp8"]), _pages(shape, gen, case["fp8"])
    s["src"] = torch.empty((R, Hkv, budget), dtype=torch.int32, device="cuda")
    s["new_lens"] = torch.empty(R, dtype=torch.int32, device="cuda")
    s["weights_out"], s["pos_out"] = torch.zeros_like(s["weights"]), torch.full_like(s["pos"], -1)
    return s


# ----------------------------------------------------------------------------- passes

def run(state):
    s = state
    if own:
        return {"append": _own_append, "attend": _own_attend, "weigh": _own_weigh, "evict": _own_evict}[s["op"]](s)
    return {"append": _plain_append, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}[s["op"]](s)


def _dims(s):
    from paper_2607_00466_amd import binding as B

    return B.attn_dims(s.get("R", 0), s["Hq"], s["Hkv"], s["D"], s["bs"], s.get("max_blocks", 1), s["num_blocks"],
                       FP8 if s["fp8"] else BF16)


@functools.lru_cache(maxsize=8)
def _workspace(R, Hq, Hkv, D):
    """The workspace that a program keeps for its batches of this shape."""
    from paper_2607_00466_amd import binding as B

    return B.attn_workspace(B.attn_dims(R, Hq, Hkv, D, 16, 1, 1))


def _own_append(s):
    from paper_2607_00466_amd import binding as B

    B.moe_kv_append(s["q"], s["k"], s["v"], s["positions"], s["pair_axis"], s["cos"], s["sin"], s["slots"], _dims(s),
                    s["q_out"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], interleaved=s["interleaved"])
    return s["q_out"], s["k_cache"], s["v_cache"]


def _own_attend(s):
    from paper_2607_00466_amd import binding as B

    B.moe_attn_decode(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["lens"], _dims(s), s["out"], s["lse"],
                      _workspace(s["R"], s["Hq"], s["Hkv"], s["D"]), group_start=s["group_start"],
                      prefix_len=s["prefix_len"], k_scale=s["k_scale"], v_scale=s["v_scale"], sinks=s["sinks"],
                      window=s["window"])
    return s["out"], s["lse"]


def _own_weigh(s):
    from paper_2607_00466_amd import binding as B

    B.moe_attn_weights(s["q"], s["k_cache"], s["block_table"], s["lens"], s["lse"], _dims(s), s["weights"],
                       s["weights_out"], group_start=s["group_start"], prefix_len=s["prefix_len"], k_scale=s["k_scale"])
    return s["weights_out"]


def _own_evict(s):
    from paper_2607_00466_amd import binding as B

    B.moe_kv_evict(s["weights"], s["pos"], s["lens"], s["seen"], s["block_table"], _dims(s), s["budget"], s["recent"],
                   s["k_cache"], s["v_cache"], s["src"], s["new_lens"], s["weights_out"], s["pos_out"],
                   protect=s["protect_rows"])
    return s["src"], s["new_lens"], s["weights_out"], s["pos_out"], s["k_cache"], s["v_cache"]


# ----------------------------------------------------------------------------- the plain forms

def _stored(x, scale, dtype):
    """fp32 values [.., Hkv, D] as the cache holds them."""
    if dtype is not FP8:
        return x.to(dtype)
    return (x / scale[:, None]).clamp(-FP8_MAX, FP8_MAX).to(FP8)


def _plain_append(s):
    rot, bs = s["rot"], s["bs"]
    at = s["positions"].long()[s["pair_axis"].long()].T  # [T, rot / 2]
    pair = torch.arange(rot // 2, device="cuda")
    c, si = s["cos"][at, pair][:, None], s["sin"][at, pair][:, None]

    def turned(x):
        x = x.float()
        if s["interleaved"]:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        else:
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        a, b = a * c - b * si, b * c + a * si
        y = torch.stack([a, b], -1).flatten(-2) if s["interleaved"] else torch.cat([a, b], -1)
        return torch.cat([y, x[..., rot:]], -1)

    s["q_out"].copy_(turned(s["q"]))
    blk, off = s["slots"].long() // bs, s["slots"].long() % bs
    for_bytes = torch.uint8 if s["fp8"] else BF16
    s["k_cache"].view(for_bytes)[blk, :, off] = _stored(turned(s["k"]), s["k_scale"], s["k_cache"].dtype).view(for_bytes)
    s["v_cache"].view(for_bytes)[blk, :, off] = _stored(s["v"].float(), s["v_scale"], s["v_cache"].dtype).view(for_bytes)
    return s["q_out"], s["k_cache"], s["v_cache"]


def _cached(s, cache, scale):
    """Each request's cached rows in fp32: [R, Hkv, longest, D]."""
    tok = torch.arange(s["longest"], device="cuda")
    blk = s["block_table"][:, tok // s["bs"]].long().clamp_min(0)
    raw = cache.view(torch.uint8) if s["fp8"] else cache
    rows = raw.transpose(1, 2)[blk, tok % s["bs"]]  # [R, longest, Hkv, D]
    rows = (rows.view(FP8) if s["fp8"] else rows).float()
    return (rows if scale is None else rows * scale[:, None]).transpose(1, 2)


def _plain_softmax(s):
    """exp(score - max), its sum over the visible tokens and the sink, and lse."""
    R, Hq, Hkv, D = s["R"], s["Hq"], s["Hkv"], s["D"]
    q = s["q"].float().view(R, Hkv, Hq // Hkv, D)
    score = torch.matmul(q, _cached(s, s["k_cache"], s["k_scale"]).transpose(2, 3)) / math.sqrt(D)
    tok = torch.arange(s["longest"], device="cuda")
    n = s["lens"][:, None]
    seen = tok < n
    if s["window"]:
        seen = seen & (tok >= n - s["window"])
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    if s["sinks"] is not None:
        sink = s["sinks"].view(Hkv, -1, 1)
        top = torch.maximum(top, sink)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    if s["sinks"] is not None:
        total = total + torch.exp(sink - top)
    return p, total, (top + total.log()).view(R, Hq)


def _plain_attend(s):
    p, total, lse = _plain_softmax(s)
    out = torch.matmul(p, _cached(s, s["v_cache"], s["v_scale"])) / total
    s["out"].copy_(out.view(s["R"], s["Hq"], s["D"]))
    s["lse"].copy_(lse)
    return s["out"], s["lse"]


def _plain_weigh(s):
    R, Hq, Hkv, D = s["R"], s["Hq"], s["Hkv"], s["D"]
    q = s["q"].float().view(R, Hkv, Hq // Hkv, D)
    score = torch.matmul(q, _cached(s, s["k_cache"], s["k_scale"]).transpose(2, 3)) / math.sqrt(D)
    p = torch.exp(score - s["lse"].view(R, Hkv, -1, 1)).sum(2)
    seen = torch.arange(s["longest"], device="cuda") < s["lens"][:, None, None]
    part = s["weights_out"][..., :s["longest"]]
    part.copy_(torch.where(seen, s["weights"][..., :s["longest"]] + p, part))
    return s["weights_out"]


def _plain_evict(s):
    R, Hkv, bs, budget = s["R"], s["Hkv"], s["bs"], s["budget"]
    N = s["weights"].shape[-1]
    n = s["lens"][:, None, None]
    slot = torch.arange(N, device="cuda", dtype=torch.int32)
    kept_for_sure = (slot < s["protect_rows"][:, None, None]) | (s["pos"] >= s["seen"][:, None, None] - s["recent"])
    key = torch.where(kept_for_sure, math.inf, s["weights"]).masked_fill(slot >= n, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :budget]
    kept = torch.zeros((R, Hkv, N), dtype=torch.bool, device="cuda").scatter_(2, order, True) & (slot < n)
    # the i-th evicted slot below the budget takes the i-th kept token past it
    hole = ~kept & (slot < torch.minimum(n, torch.tensor(budget, device="cuda")))
    mover = kept & (slot >= budget)
    movers = torch.sort((~mover).to(torch.uint8), dim=-1, stable=True).indices  # kept ones past the budget first
    nth = (hole.int().cumsum(-1) - 1).clamp_min(0)
    src = torch.where(hole, movers.gather(2, nth.long()).to(torch.int32), slot)
    src = torch.where(slot < n, src, -1)[..., :budget]
    src = torch.nn.functional.pad(src, (0, budget - src.shape[-1]), value=-1)
    s["src"].copy_(src)
    torch.minimum(s["lens"], torch.tensor(budget, device="cuda", dtype=torch.int32), out=s["new_lens"])
    full = torch.nn.functional.pad(src, (0, N))[..., :N].clamp_min(0).long()
    left = slot < s["new_lens"][:, None, None]
    s["weights_out"].copy_(torch.where(slot < n, torch.where(left, s["weights"].gather(2, full), 0.0), s["weights_out"]))
    s["pos_out"].copy_(torch.where(slot < n, torch.where(left, s["pos"].gather(2, full), -1), s["pos_out"]))
    # the moved rows, every page offset by its table
    r, h, i = (hole & (slot < budget)).nonzero(as_tuple=True)
    j = full[r, h, i]
    table = s["block_table"].long()
    to, at = table[r, i // bs], table[r, j // bs]
    raw = torch.uint8 if s["fp8"] else BF16
    k, v = s["k_cache"].view(raw), s["v_cache"].view(raw)
    k[to, h, i % bs] = k[at, h, j % bs]
    v[to, h, i % bs] = v[at, h, j % bs]
    return s["src"], s["new_lens"], s["weights_out"], s["pos_out"], s["k_cache"], s["v_cache"]


# ----------------------------------------------------------------------------- 64 bits, from the definitions

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attn, "weigh": _exact_attn, "evict": _exact_evict}[case["op"]](s)


def _exact_append(s):
    """The rotation as a product of complex numbers, rows written one by one."""
    T, rot, bs = s["T"], s["rot"], s["bs"]
    i = torch.arange(rot // 2, device="cuda")
    at = torch.stack([s["positions"][a] for a in s["pair_axis"].tolist()], 1).long()
    turn = torch.complex(s["cos"].double()[at, i], s["sin"].double()[at, i])[:, None]
    lower = 2 * i if s["interleaved"] else i
    upper = lower + (1 if s["interleaved"] else rot // 2)

    def turned(x):
        y = x.double().clone()
        z = torch.complex(y[..., lower], y[..., upper]) * turn
        y[..., lower], y[..., upper] = z.real, z.imag
        return y

    q, k, v = turned(s["q"]), turned(s["k"]), s["v"].double()
    caches = []
    for x, scale in ((k, s["k_scale"]), (v, s["v_scale"])):
        if scale is not None:
            x = (x / scale.double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
        cache = torch.zeros(s["k_cache"].shape, dtype=torch.float64, device="cuda")
        for t, slot in enumerate(s["slots"].tolist()):
            cache[slot // bs, :, slot % bs] = x[t]
        caches.append(cache)
    return q, caches[0], caches[1]


def _exact_attn(s):
    """Request by request, over its own rows alone."""
    R, Hq, Hkv, D, bs = (s[k] for k in ("R", "Hq", "Hkv", "D", "bs"))
    G = Hq // Hkv
    out, lses = torch.zeros((R, Hq, D), dtype=torch.float64, device="cuda"), torch.empty((R, Hq), dtype=torch.float64, device="cuda")
    weights = s["weights_out"].double() if s["op"] == "weigh" else None
    for r, n in enumerate(s["lens"].tolist()):
        lo = max(0, n - s["window"]) if s["window"] else 0
        blk = s["block_table"][r, :-(-n // bs)].long()

        def rows(cache, scale):
            x = cache[blk].double() if not s["fp8"] else cache.view(torch.uint8)[blk].view(FP8).double()
            x = x.transpose(0, 1).reshape(Hkv, -1, D)[:, lo:n]
            return x if scale is None else x * scale.double()[:, None, None]

        score = rows(s["k_cache"], s["k_scale"]) @ s["q"][r].double().view(Hkv, G, D).transpose(1, 2).contiguous()
        score = score.transpose(1, 2).reshape(Hq, n - lo) * D ** -0.5
        if s["op"] == "weigh":
            p = torch.exp(score - s["lse"][r].double()[:, None]).view(Hkv, G, n)
            weights[r, :, :n] = s["weights"][r, :, :n].double() + p.sum(1)
            continue
        every = score if s["sinks"] is None else torch.cat([score, s["sinks"].double()[:, None]], 1)
        lses[r] = torch.logsumexp(every, 1)
        p = torch.exp(score - lses[r][:, None]).view(Hkv, G, n - lo)
        out[r] = (p @ rows(s["v_cache"], s["v_scale"])).view(Hq, D)
    return weights if s["op"] == "weigh" else (out, lses)


def _exact_evict(s):
    """Row by row on the host: rank the slots, then fill the holes in order."""
    R, Hkv, bs, budget = (s[k] for k in ("R", "Hkv", "bs", "budget"))
    weights, pos = s["weights"].double().cpu().numpy(), s["pos"].cpu().numpy()
    w_out, p_out = s["weights_out"].double().cpu().numpy(), s["pos_out"].cpu().numpy()
    src = np.full((R, Hkv, budget), -1, np.int32)
    lens, seen, protect = (s[k].tolist() for k in ("lens", "seen", "protect_rows"))
    for r in range(R):
        n = lens[r]
        for h in range(Hkv):
            slots = np.arange(n)
            sure = (slots < protect[r]) | (pos[r, h, :n] >= seen[r] - s["recent"])
            best = np.lexsort((slots, -weights[r, h, :n], ~sure))[:budget]
            stays = np.zeros(n, bool)
            stays[best] = True
            at = np.arange(min(n, budget))
            at[~stays[:budget]] = budget + np.flatnonzero(stays[budget:])
            src[r, h, :len(at)] = at
            w_out[r, h, :n], p_out[r, h, :n] = 0.0, -1
            w_out[r, h, :len(at)], p_out[r, h, :len(at)] = weights[r, h, at], pos[r, h, at]
    # the caches as the list of sources says, from copies of what they held
    r, h, i = np.nonzero((src >= 0) & (src != np.arange(budget)))
    r, h, i, j = (torch.from_numpy(np.asarray(x, np.int64)).cuda() for x in (r, h, i, src[r, h, i]))
    table = s["block_table"].long()
    caches = []
    for cache in (s["k_cache"], s["v_cache"]):
        held = cache.double()
        after = held.clone()
        after[table[r, i // bs], h, i % bs] = held[table[r, j // bs], h, j % bs]
        caches.append(after)
    return src, np.minimum(np.asarray(lens, np.int32), budget).astype(np.int32), w_out, p_out, caches[0], caches[1]
