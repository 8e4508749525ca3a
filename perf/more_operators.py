"""What a decode worker's paged cache needs beside append and attention: what is measured of its operators.

Four operators:

  norm     queries and keys normed head by head and turned by their positions in one pass,
           keys and values written to their pages (bf16 or fp8)
  quantise the same (norms or none) into a cache of 8-bit integers with a scale for each page
           and kv head: the runs of new tokens of several requests, pages partly filled before
  attend   one query token a request against that cache; prefixes that requests share read
           once for the group, sinks, windows
  pages    fork: a request's copy that shares its full pages and gets the last one for itself;
           compact: live pages move into free ones, block tables follow; in all layers at once

``run`` computes them by elementary torch operations, or, where ``own`` is true, by the
library's entry points.  Shapes are those of the decode layers this repository names
(batches of 1 to 256 requests; 32 query heads over 4 of 128, 64 over 8 of 64, block size 16,
48 layers) and generic ones near them.

A cache of 8-bit integers is returned as its codes, whole numbers, with the scales beside them.
"""
import math
import random

import torch

own = False

BF16, FP8, INT8 = torch.bfloat16, torch.float8_e4m3fn, torch.int8
FP8_MAX, INT8_MAX = 448.0, 127.0
EPS = 1e-6


# ----------------------------------------------------------------------------- cases

def _norm(name, T, Hq, Hkv, D, rot, interleaved=False, fp8=False, fp32=False, bs=16):
    """T new tokens: queries and keys normed and rotated, keys and values written to their pages."""
    return dict(name=name, op="norm", T=T, Hq=Hq, Hkv=Hkv, D=D, rot=rot, interleaved=interleaved, fp8=fp8,
                fp32=fp32, bs=bs)


def _quantise(name, R, lo, hi, held, Hq, Hkv, D, rot, norms=True, interleaved=False, fp32=False, bs=16):
    """lo to hi new tokens of each of R requests that hold up to ``held`` already."""
    return dict(name=name, op="quantise", R=R, lo=lo, hi=hi, held=held, Hq=Hq, Hkv=Hkv, D=D, rot=rot, norms=norms,
                interleaved=interleaved, fp32=fp32, bs=bs)


def _attend(name, R, Hq, Hkv, D, lo, hi, groups=0, prefix=0, window=0, sinks=False, bs=16):
    """R requests with lo to hi cached tokens of their own each, after a prefix of
    ``prefix`` tokens that each of ``groups`` equal groups shares."""
    return dict(name=name, op="attend", R=R, Hq=Hq, Hkv=Hkv, D=D, lo=lo, hi=hi, groups=groups, prefix=prefix,
                window=window, sinks=sinks, bs=bs)


def _fork(name, parents, each, layers, Hkv, D, held, kv, bs=16):
    """``each`` copies of each of ``parents`` requests of up to ``held`` tokens, in all layers."""
    return dict(name=name, op="fork", parents=parents, each=each, layers=layers, Hkv=Hkv, D=D, held=held, kv=kv, bs=bs)


def _compact(name, R, held, free, layers, Hkv, D, kv, bs=16):
    """The pages of R requests of up to ``held`` tokens, scattered among ``free`` as many
    free ones again, moved together."""
    return dict(name=name, op="compact", R=R, held=held, free=free, layers=layers, Hkv=Hkv, D=D, kv=kv, bs=bs)


def listed():
    return [
        # the new token of each request of a decode batch: latency counts
        _norm("norm 64 new tokens", 64, 32, 4, 128, 128),
        # an odd long prompt with activations in fp32, into an fp8 cache
        _norm("norm 4097 from fp32 to fp8", 4097, 32, 4, 128, 128, fp32=True, fp8=True),
        # a decode batch, whose pages are partly filled: latency counts
        _quantise("quantise 64 new tokens", 64, 1, 1, 200, 32, 4, 128, 128),
        # a batch of prompts, some behind tokens that are cached already
        _quantise("quantise 16 prompts", 16, 1, 1000, 50, 64, 8, 64, 64, norms=False, fp32=True),
        # few requests, short contexts: latency counts
        _attend("attend 8 of up to 512", 8, 32, 4, 128, 1, 512),
        # an ordinary batch of mixed lengths, nothing shared
        _attend("attend 128 of up to 8000", 128, 32, 4, 128, 17, 8000),
        # two requests with very long contexts: the work of a row split over the chip
        _attend("attend 2 near 131000", 2, 32, 4, 128, 129999, 131071),
        # a large batch of several domains, 64-wide heads with sink logits
        _attend("attend 256 behind 8 x 2048", 256, 64, 8, 64, 1, 1500, groups=8, prefix=2048, sinks=True),
        # a few requests sampled once more, one layer: latency counts
        _fork("fork 4 in 1 layer", 4, 1, 1, 4, 128, 200, "bf16"),
        # several answers to each of a batch's prompts, in all layers
        _fork("fork 16 x 4 in 48 layers", 16, 4, 48, 4, 128, 300, "int8"),
        # few pages, one layer
        _compact("compact 4 requests", 4, 300, 1.0, 1, 8, 64, "bf16"),
        # a batch that shrank, its pages moved together in all layers
        _compact("compact 32 requests in 48 layers", 32, 500, 1.0, 48, 4, 128, "int8"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    Hq, Hkv, D = rng.choice([(32, 4, 128), (64, 8, 64), (32, 8, 128), (16, 16, 64), (20, 4, 128), (16, 2, 256)])
    bs = rng.choice([16, 16, 32, 64])
    op = rng.choice(["norm", "quantise", "attend", "attend", "fork", "compact"])
    if op == "norm":
        c = _norm("", min(_log(rng, 1, 4097), 4097 * 4608 // ((Hq + 2 * Hkv) * D)), Hq, Hkv, D, rng.choice([D, D, D // 2, 32]),
                  interleaved=rng.random() < 0.3, fp8=rng.random() < 0.5, fp32=rng.random() < 0.4, bs=bs)
    elif op == "quantise":
        R = _log(rng, 1, 256)
        hi = _log(rng, 1, max(1, 6000 * 4608 // (R * (Hq + 2 * Hkv) * D)))
        c = _quantise("", R, max(1, hi // rng.choice([1, 2, 50])), hi, _log(rng, 1, 300), Hq, Hkv, D, rng.choice([D, D, D // 2]),
                      norms=rng.random() < 0.6, interleaved=rng.random() < 0.3, fp32=rng.random() < 0.4, bs=bs)
    elif op == "attend":
        shared = rng.random() < 0.5
        R = _log(rng, 2 if shared else 1, 256)
        if R > 64 and D == 256:
            Hq, Hkv, D = 32, 8, 128
        groups = rng.choice([1, 1, max(1, R // 16), max(1, R // 3)]) if shared else 0
        # no more products and no more cached bytes than the largest of the listed
        longest = min(8192, 2000000000 // (R * Hq * D))
        prefix = bs * max(1, _log(rng, min(64, longest), longest) // bs) if shared else 0
        rows = (100000000 if shared else 250000000) // (Hkv * D)
        hi = _log(rng, 1, min(131000, max(64, rows // R)))
        plain = not shared and rng.random() < 0.25
        c = _attend("", R, Hq, Hkv, D, max(1, hi // rng.choice([1, 4, 64])), hi, groups, prefix,
                    window=_log(rng, 16, 1024) if plain else 0, sinks=rng.random() < 0.3, bs=bs)
    else:
        kv, layers = rng.choice(["bf16", "fp8", "int8"]), _log(rng, 1, 48)
        if op == "fork":
            parents = _log(rng, 1, 32)
            c = _fork("", parents, _log(rng, 1, max(1, 64 // parents)), max(1, min(layers, 1600000 // (bs * Hkv * D))), Hkv, D,
                      _log(rng, 1, 300), kv, bs)
        else:
            R = _log(rng, 1, 32)
            c = _compact("", R, _log(rng, 16, 500), rng.choice([0.25, 1.0, 2.0]), max(1, min(layers, 12000 // (Hkv * D))), Hkv, D, kv, bs)
    del c["name"]
    return c


def _between(case, lo, hi, n, what):
    """n numbers of lo to hi: a fixed draw for the case, its end among them."""
    r = random.Random("%s %d %d %d" % (what, lo, hi, n))
    got = [r.randint(lo, hi) for _ in range(n)]
    got[-1] = hi
    return got


def _lens(case):
    return _between(case, case["lo"], case["hi"], case["R"], "lens")


def _bounds(case):
    """The groups' first requests, and R."""
    return [g * case["R"] // case["groups"] for g in range(case["groups"] + 1)]


def _elem(kv):
    return 2 if kv == "bf16" else 1


def work(case):
    c = case
    if c["op"] in ("norm", "quantise"):
        T = c["T"] if c["op"] == "norm" else sum(_lens(c))
        e = 1 if c["op"] == "quantise" or c["fp8"] else 2
        rows = T * c["D"]
        n_in = (c["Hq"] + 2 * c["Hkv"]) * rows * (4 if c["fp32"] else 2)
        more = 0
        if c["op"] == "quantise":  # the scales of the pages that receive tokens
            more = 16 * c["Hkv"] * sum(-(-(h % c["bs"] + n) // c["bs"]) for h, n in zip(_held(c), _lens(c)))
        return {"bytes": n_in + c["Hq"] * rows * 2 + 2 * c["Hkv"] * rows * e + 4 * T * (2 + c["rot"]) + more,
                "flops": 7 * T * (c["Hq"] + c["Hkv"]) * c["D"]}
    if c["op"] == "attend":
        lens = _lens(c)
        kept = [min(n, c["window"]) if c["window"] else n for n in lens]
        distinct = sum(kept) + c["groups"] * c["prefix"]
        seen = sum(kept) + c["R"] * c["prefix"]
        pages = sum(-(-n // c["bs"]) for n in kept) + c["groups"] * c["prefix"] // c["bs"]
        return {"bytes": distinct * 2 * c["Hkv"] * c["D"] + pages * (8 * c["Hkv"] + 4) + c["R"] * c["Hq"] * (4 * c["D"] + 4),
                "flops": 4 * seen * c["Hq"] * c["D"]}
    row = 2 * c["Hkv"] * c["D"] * _elem(c["kv"]) * c["layers"]  # a token's keys and values
    scales = 8 * c["Hkv"] * c["layers"] if c["kv"] == "int8" else 0
    lens = _parents(c) if c["op"] == "fork" else _between(c, max(1, c["held"] // 4), c["held"], c["R"], "compact")
    width = max(-(-n // c["bs"]) for n in lens)
    if c["op"] == "fork":
        rest = [n % c["bs"] for n in lens]
        return {"bytes": c["each"] * (2 * row * sum(rest) + 2 * scales * sum(n > 0 for n in rest) + 8 * width * len(lens)), "flops": 0}
    live = sum(-(-n // c["bs"]) for n in lens)
    nb = live + int(live * c["free"]) + 1
    # of the live pages, the share past the first `live` places moves
    moved = live * (1 - live / nb)
    return {"bytes": int(2 * moved * (row * c["bs"] + scales)) + 8 * width * len(lens) + 4 * nb, "flops": 0}


def _held(case):
    """Tokens that the requests hold before the new ones."""
    return _between(case, 0, case["held"], case["R"], "held")


def _parents(case):
    return _between(case, max(1, case["held"] // 3), case["held"], case["parents"], "fork")


# ----------------------------------------------------------------------------- inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = random.Random(seed)
    return {"norm": _prepare_norm, "quantise": _prepare_quantise, "attend": _prepare_attend, "fork": _prepare_fork,
            "compact": _prepare_compact}[case["op"]](case, gen, host)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _quantised(x):
    """Values as codes and a scale for each page and head: (int8 like x, fp32)."""
    scale = x.abs().amax((-2, -1), keepdim=True).float() / INT8_MAX
    return torch.round(x / scale).to(INT8), scale.squeeze(-1).squeeze(-1).contiguous()


def _pages(shape, gen, kv):
    """Random pages [.., Hkv, bs, D], and their scales: of each page and head where kv is
    int8, of each head where it is fp8."""
    x = torch.empty(shape, dtype=BF16, device="cuda").normal_(0, 1, generator=gen)
    if kv == "int8":
        return _quantised(x)
    if kv == "fp8":
        return x.to(FP8), 0.5 + torch.rand(shape[-3], device="cuda", generator=gen)
    return x, None


def _projected(case, T, gen):
    """Queries, keys and values as one projection leaves them: views of its rows.  Heads of
    different size, as trained ones are."""
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    qkv = torch.empty((T, Hq + 2 * Hkv, D), device="cuda").normal_(generator=gen)
    qkv *= torch.empty(Hq + 2 * Hkv, 1, device="cuda").uniform_(0.2, 4.0, generator=gen)
    qkv = qkv if case["fp32"] else qkv.to(BF16)
    return dict(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], q_out=torch.zeros((T, Hq, D), device="cuda", dtype=BF16))


def _turns(case, gen):
    rot, D = case["rot"], case["D"]
    freq = 1e6 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / rot)
    angle = torch.arange(40960, device="cuda", dtype=torch.float64)[:, None] * freq
    norms = case.get("norms", True)
    weights = [1 + 0.2 * torch.empty(D, device="cuda").normal_(generator=gen) if norms else None for _ in "qk"]
    return dict(cos=angle.cos().float(), sin=angle.sin().float(), q_norm=weights[0], k_norm=weights[1],
                pair_axis=torch.zeros(rot // 2, dtype=torch.int32, device="cuda"))


def _prepare_norm(case, gen, host):
    T, Hkv, D, bs = (case[k] for k in ("T", "Hkv", "D", "bs"))
    s = dict(case, **_projected(case, T, gen), **_turns(case, gen))
    # a prompt's positions, or a decode batch's
    if T > 256:
        s["positions"] = torch.arange(T, device="cuda", dtype=torch.int32)[None] + host.randrange(30000)
    else:
        s["positions"] = torch.randint(0, 40960, (1, T), device="cuda", dtype=torch.int32, generator=gen)
    s["num_blocks"] = -(-T // bs) + 7
    blocks = torch.randperm(s["num_blocks"], device="cuda", generator=gen)
    i = torch.arange(T, device="cuda")
    s["slots"] = (blocks[i // bs] * bs + i % bs).to(torch.int32)
    s["k_scale"], s["v_scale"] = (0.05 + 0.05 * torch.rand(Hkv, device="cuda", generator=gen) if case["fp8"] else None for _ in "kv")
    shape = (s["num_blocks"], Hkv, bs, D)
    s["k_cache"], s["v_cache"] = (torch.zeros(shape, device="cuda", dtype=BF16).to(FP8 if case["fp8"] else BF16) for _ in "kv")
    return s


def _tables(blocks, host, spare):
    """Block tables [len(blocks), widest] over scattered pages, blocks[r] of row r."""
    nb = sum(blocks) + spare
    ids = list(range(nb))
    host.shuffle(ids)
    rows = [[ids.pop() for _ in range(n)] for n in blocks]
    width = max(1, max(blocks))
    return [t + [-1] * (width - len(t)) for t in rows], nb, width, ids


def _prepare_quantise(case, gen, host):
    R, Hkv, D, bs = (case[k] for k in ("R", "Hkv", "D", "bs"))
    new, held = _lens(case), _held(case)
    T = sum(new)
    s = dict(case, T=T, **_projected(case, T, gen), **_turns(case, gen))
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    s["query_start"], s["lens"] = _i32(start), _i32(held)
    s["positions"] = torch.cat([torch.arange(h, h + n, device="cuda", dtype=torch.int32) for h, n in zip(held, new)])[None]
    table, s["num_blocks"], s["max_blocks"], _ = _tables([-(-(h + n) // bs) for h, n in zip(held, new)], host, 7)
    s["block_table"] = _i32(table)
    # what the pages hold before is quieter than some of what comes: their scales grow
    shape = (s["num_blocks"], Hkv, bs, D)
    for which in "kv":
        codes, scale = _pages(shape, gen, "int8")
        s[which + "_cache"], s[which + "_scale"] = codes, scale * torch.empty_like(scale).uniform_(0.1, 1.5, generator=gen)
    return s


def _prepare_attend(case, gen, host):
    R, Hq, Hkv, D, bs, prefix = (case[k] for k in ("R", "Hq", "Hkv", "D", "bs", "prefix"))
    s = dict(case)
    lens = _lens(case)
    groups = _bounds(case) if case["groups"] else []
    table, nb, width, ids = _tables([-(-n // bs) for n in lens], host, len(groups[1:]) * (prefix // bs) + 5)
    if groups:
        shared = [[ids.pop() for _ in range(prefix // bs)] for _ in groups[1:]]
        table = [shared[next(g for g in range(len(shared)) if groups[g] <= r < groups[g + 1])] + t for r, t in enumerate(table)]
        width += prefix // bs
    s["block_table"], s["num_blocks"], s["max_blocks"] = _i32(table), nb, width
    total = [n + prefix for n in lens]
    s["longest"], s["lens"] = max(total), _i32(total)
    s["group_start"] = _i32(groups) if groups else None
    s["prefix_len"] = torch.full((case["groups"],), prefix, dtype=torch.int32, device="cuda") if groups else None
    shape = (nb, Hkv, bs, D)
    s["k_cache"], s["k_scale"] = _pages(shape, gen, "int8")
    s["v_cache"], s["v_scale"] = _pages(shape, gen, "int8")
    # scores of spread 2: some tokens stand out, as they do in a trained model
    s["q"] = torch.empty((R, Hq, D), dtype=BF16, device="cuda").normal_(0, 2, generator=gen)
    s["sinks"] = torch.empty(Hq, device="cuda").normal_(2, 1, generator=gen) if case["sinks"] else None
    s["out"] = torch.empty((R, Hq, D), dtype=BF16, device="cuda")
    s["lse"] = torch.empty((R, Hq), dtype=torch.float32, device="cuda")
    return s


def _layered(s, case, gen):
    shape = (case["layers"], s["num_blocks"], case["Hkv"], case["bs"], case["D"])
    s["k_cache"], s["k_scale"] = _pages(shape, gen, case["kv"])
    s["v_cache"], s["v_scale"] = _pages(shape, gen, case["kv"])
    if case["kv"] == "fp8":  # the heads' scales stay with the layer, not with the pages
        s["k_scale"] = s["v_scale"] = None
    return s


def _prepare_fork(case, gen, host):
    bs, each = case["bs"], case["each"]
    lens = _parents(case)
    n = len(lens)
    s = dict(case, R=n * (1 + each))
    blocks = [-(-k // bs) for k in lens]
    table, s["num_blocks"], s["max_blocks"], ids = _tables(blocks, host, n * each + 5)
    # rows of the copies: empty requests' so far
    s["block_table"] = _i32(table + [[-1] * s["max_blocks"]] * (n * each))
    s["lens"] = _i32(lens + [0] * (n * each))
    s["parent"] = _i32([p for p in range(n) for _ in range(each)])
    s["child"] = _i32(list(range(n, n * (1 + each))))
    s["page"] = _i32([ids.pop() for _ in range(n * each)])
    return _layered(s, case, gen)


def _prepare_compact(case, gen, host):
    bs = case["bs"]
    lens = _between(case, max(1, case["held"] // 4), case["held"], case["R"], "compact")
    blocks = [-(-k // bs) for k in lens]
    live = sum(blocks)
    s = dict(case)
    table, s["num_blocks"], s["max_blocks"], ids = _tables(blocks, host, int(live * case["free"]) + 1)
    free = sorted(b for b in ids if b < live)
    remap = [-1] * s["num_blocks"]
    for row in table:
        for b in row:
            if b >= 0:
                remap[b] = b
    movers = [b for b in range(live, s["num_blocks"]) if remap[b] == b]
    for b, to in zip(movers, free):
        remap[b] = to
    s["block_table"], s["remap"] = _i32(table), _i32(remap)
    s["table_out"] = torch.zeros_like(s["block_table"])
    return _layered(s, case, gen)


# ----------------------------------------------------------------------------- passes

def run(state):
    s = state
    if own:
        return {"norm": _own_norm, "quantise": _own_quantise, "attend": _own_attend, "fork": _own_fork,
                "compact": _own_compact}[s["op"]](s)
    return {"norm": _plain_norm, "quantise": _plain_quantise, "attend": _plain_attend, "fork": _plain_fork,
            "compact": _plain_compact}[s["op"]](s)


def _dims(s, kv):
    from paper_2607_00466_amd import binding as B

    return B.attn_dims(s.get("R", 0), s.get("Hq", s["Hkv"]), s["Hkv"], s["D"], s["bs"], s.get("max_blocks", 1), s["num_blocks"], kv)


def _workspace(s, d):
    """The workspace that a program keeps for its batches of this shape: one a state, since
    calls on two streams cannot share one, nor calls on two devices."""
    from paper_2607_00466_amd import binding as B

    if "ws" not in s:
        s["ws"] = B.attn_workspace(d, s["q"].device)
    return s["ws"]


def _own_norm(s):
    from paper_2607_00466_amd import binding as B

    B.moe_kv_append_norm(s["q"], s["k"], s["v"], s["positions"], s["pair_axis"], s["cos"], s["sin"], s["slots"],
                         _dims(s, FP8 if s["fp8"] else BF16), s["q_out"], s["k_cache"], s["v_cache"], s["q_norm"], s["k_norm"],
                         eps=EPS, k_scale=s["k_scale"], v_scale=s["v_scale"], interleaved=s["interleaved"])
    return s["q_out"], s["k_cache"], s["v_cache"]


def _own_quantise(s):
    from paper_2607_00466_amd import binding as B

    B.moe_kv_append_int8(s["q"], s["k"], s["v"], s["positions"], s["pair_axis"], s["cos"], s["sin"], s["query_start"],
                         s["block_table"], s["lens"], _dims(s, INT8), s["q_out"], s["k_cache"], s["v_cache"], s["k_scale"],
                         s["v_scale"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS, interleaved=s["interleaved"])
    return s["q_out"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]


def _own_attend(s):
    from paper_2607_00466_amd import binding as B

    d = _dims(s, INT8)
    B.moe_attn_decode(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["lens"], d, s["out"], s["lse"],
                      _workspace(s, d), group_start=s["group_start"],
                      prefix_len=s["prefix_len"], k_scale=s["k_scale"], v_scale=s["v_scale"], sinks=s["sinks"],
                      window=s["window"])
    return s["out"], s["lse"]


def _changed(s):
    return tuple(s[k] for k in ("k_cache", "v_cache", "k_scale", "v_scale") if s[k] is not None)


def _kv(s):
    return {"bf16": BF16, "fp8": FP8, "int8": INT8}[s["kv"]]


def _own_fork(s):
    from paper_2607_00466_amd import binding as B

    B.moe_kv_fork(s["parent"], s["child"], s["page"], s["block_table"], s["lens"], _dims(s, _kv(s)), s["k_cache"],
                  s["v_cache"], s["k_scale"], s["v_scale"])
    return s["block_table"], s["lens"], _changed(s)


def _own_compact(s):
    from paper_2607_00466_amd import binding as B

    B.moe_kv_compact(s["remap"], s["block_table"], s["table_out"], _dims(s, _kv(s)), s["k_cache"], s["v_cache"],
                     s["k_scale"], s["v_scale"])
    return s["table_out"], _changed(s)


# ----------------------------------------------------------------------------- the plain forms

def _normed(x, weight):
    """Each head over the root of its mean square, in fp32; the mean in 64 bits, since codes
    next to a border turn on the last bit."""
    x = x.float()
    if weight is None:
        return x
    return x * (x.double().square().mean(-1, keepdim=True) + EPS).rsqrt().float() * weight


def _turned(s, x):
    """x [T, heads, D] in fp32 turned by the tokens' positions."""
    rot = s["rot"]
    at = s["positions"].long()[s["pair_axis"].long()].T  # [T, rot / 2]
    pair = torch.arange(rot // 2, device="cuda")
    c, si = s["cos"][at, pair][:, None], s["sin"][at, pair][:, None]
    if s["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    a, b = a * c - b * si, b * c + a * si
    y = torch.stack([a, b], -1).flatten(-2) if s["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_norm(s):
    bs = s["bs"]
    s["q_out"].copy_(_turned(s, _normed(s["q"], s["q_norm"])))
    blk, off = s["slots"].long() // bs, s["slots"].long() % bs
    raw = torch.uint8 if s["fp8"] else BF16
    for x, which in ((_turned(s, _normed(s["k"], s["k_norm"])), "k"), (s["v"].float(), "v")):
        if s["fp8"]:
            x = (x / s[which + "_scale"][:, None]).clamp(-FP8_MAX, FP8_MAX)
        s[which + "_cache"].view(raw)[blk, :, off] = x.to(s[which + "_cache"].dtype).view(raw)
    return s["q_out"], s["k_cache"], s["v_cache"]


def _plain_quantise(s):
    bs, nb = s["bs"], s["num_blocks"]
    s["q_out"].copy_(_turned(s, _normed(s["q"], s["q_norm"])))
    t = torch.arange(s["T"], device="cuda")
    r = torch.searchsorted(s["query_start"].long(), t, right=True) - 1
    j = s["lens"].long()[r] + t - s["query_start"].long()[r]
    page, off = s["block_table"].long()[r, j // bs], j % bs
    # each page's first new token: earlier ones are held
    first = torch.full((nb,), bs, device="cuda").scatter_reduce(0, page, off, "amin")[:, None]
    touched, held = first < bs, (first > 0) & (first < bs)
    for x, which in ((_turned(s, _normed(s["k"], s["k_norm"])), "k"), (s["v"].float(), "v")):
        codes, scale = s[which + "_cache"], s[which + "_scale"]
        top = torch.zeros_like(scale).scatter_reduce(0, page[:, None].expand(-1, s["Hkv"]), x.abs().amax(-1), "amax")
        # a page that holds tokens doubles its scale as often as the new ones need
        m, e = torch.frexp(top.double() / (INT8_MAX * scale.double()))
        more = torch.where(m > 0.5, e, e - 1).clamp_min(0)
        grows = held & (scale > 0)
        after = torch.where(touched, torch.where(grows, torch.ldexp(scale, more), top / INT8_MAX), scale)
        back = torch.where(grows, scale / after, 1.0)
        row = torch.arange(bs, device="cuda")
        again = (held & (row < first))[:, None, :, None]
        codes.copy_(torch.where(again, torch.round(codes * back[:, :, None, None]), codes.float()))
        codes[page, :, off] = torch.round(x / after[page][..., None]).clamp(-INT8_MAX, INT8_MAX).to(INT8)
        scale.copy_(after)
    return s["q_out"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]


def _cached(s, cache, scale):
    """Each request's cached rows in fp32: [R, Hkv, longest, D]."""
    tok = torch.arange(s["longest"], device="cuda")
    blk = s["block_table"][:, tok // s["bs"]].long().clamp_min(0)
    rows = cache.transpose(1, 2)[blk, tok % s["bs"]]  # [R, longest, Hkv, D]
    return (rows * scale[blk][..., None]).transpose(1, 2)


def _plain_attend(s):
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
    out = torch.matmul(p, _cached(s, s["v_cache"], s["v_scale"])) / total
    s["out"].copy_(out.view(R, Hq, D))
    s["lse"].copy_((top + total.log()).view(R, Hq))
    return s["out"], s["lse"]


def _plain_fork(s):
    bs = s["bs"]
    p, c, page = s["parent"].long(), s["child"].long(), s["page"].long()
    n = s["lens"][p].long()
    full, rest = n // bs, n % bs
    i = torch.arange(s["max_blocks"], device="cuda")
    row = torch.where(i < full[:, None], s["block_table"][p], -1)
    last = s["block_table"][p].long().gather(1, full.clamp_max(s["max_blocks"] - 1)[:, None])[:, 0]
    last = torch.where(rest > 0, last, page)  # (a page copied to itself where none is partly filled)
    s["block_table"][c] = torch.where((i == full[:, None]) & (rest > 0)[:, None], s["page"][:, None], row)
    s["lens"][c] = s["lens"][p]
    keep = (torch.arange(bs, device="cuda") < rest[:, None])[:, None, :, None]
    raw = BF16 if s["kv"] == "bf16" else torch.uint8
    for which in ("k_cache", "v_cache"):
        x = s[which].view(raw)
        x[:, page] = torch.where(keep, x[:, last], x[:, page])
    if s["kv"] == "int8":
        for which in ("k_scale", "v_scale"):
            s[which][:, page] = s[which][:, last]
    return s["block_table"], s["lens"], _changed(s)


def _plain_compact(s):
    remap = s["remap"].long()
    src = ((remap >= 0) & (remap != torch.arange(s["num_blocks"], device="cuda"))).nonzero()[:, 0]
    dst = remap[src]
    raw = BF16 if s["kv"] == "bf16" else torch.uint8
    for which in ("k_cache", "v_cache"):
        x = s[which].view(raw)
        x[:, dst] = x[:, src]
    if s["kv"] == "int8":
        for which in ("k_scale", "v_scale"):
            s[which][:, dst] = s[which][:, src]
    old = s["block_table"].long()
    s["table_out"].copy_(torch.where(old >= 0, s["remap"][old.clamp_min(0)], -1))
    return s["table_out"], _changed(s)


# ----------------------------------------------------------------------------- 64 bits, from the definitions

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "quantise": _exact_quantise, "attend": _exact_attend, "fork": _exact_copies,
            "compact": _exact_copies}[case["op"]](s)


def _exact_rows(s, x, weight):
    """Normed, and the rotation as a product of complex numbers."""
    x = x.double()
    if weight is not None:
        x = weight.double() * x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / s["D"] + EPS)
    i = torch.arange(s["rot"] // 2, device="cuda")
    at = s["positions"][0].long()[:, None]
    turn = torch.complex(s["cos"].double()[at, i], s["sin"].double()[at, i])[:, None]
    lower = 2 * i if s["interleaved"] else i
    upper = lower + (1 if s["interleaved"] else s["rot"] // 2)
    y = x.clone()
    z = torch.complex(x[..., lower], x[..., upper]) * turn
    y[..., lower], y[..., upper] = z.real, z.imag
    return y


def _exact_norm(s):
    """Rows written one by one."""
    bs = s["bs"]
    caches = []
    for x, scale in ((_exact_rows(s, s["k"], s["k_norm"]), s["k_scale"]), (s["v"].double(), s["v_scale"])):
        if scale is not None:
            x = (x / scale.double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
        cache = torch.zeros(s["k_cache"].shape, dtype=torch.float64, device="cuda")
        for t, slot in enumerate(s["slots"].tolist()):
            cache[slot // bs, :, slot % bs] = x[t]
        caches.append(cache)
    return _exact_rows(s, s["q"], s["q_norm"]), caches[0], caches[1]


def _exact_quantise(s):
    """The scales, page by page; codes are whole numbers, whose borders 64 bits do not decide."""
    bs = s["bs"]
    start, held, table = s["query_start"].tolist(), s["lens"].tolist(), s["block_table"].tolist()
    scales = []
    for x, scale in ((_exact_rows(s, s["k"], s["k_norm"]), s["k_scale"]), (s["v"].double(), s["v_scale"])):
        top = x.abs().amax(-1).cpu()
        after = scale.double().cpu()
        for r in range(s["R"]):
            j, end = held[r], held[r] + start[r + 1] - start[r]
            while j < end:
                stop = min(end, (j // bs + 1) * bs)
                need = top[start[r] + j - held[r]:start[r] + stop - held[r]].amax(0) / INT8_MAX
                for h in range(s["Hkv"]):
                    a, old = float(need[h]), float(after[table[r][j // bs], h])
                    if j % bs and old > 0:
                        while old < a:
                            old *= 2
                        a = old
                    after[table[r][j // bs], h] = a
                j = stop
        scales.append(after.cuda())
    return _exact_rows(s, s["q"], s["q_norm"]), None, None, scales[0], scales[1]


def _exact_attend(s):
    """Request by request, over its own rows alone."""
    R, Hq, Hkv, D, bs = (s[k] for k in ("R", "Hq", "Hkv", "D", "bs"))
    G = Hq // Hkv
    out, lses = torch.zeros((R, Hq, D), dtype=torch.float64, device="cuda"), torch.empty((R, Hq), dtype=torch.float64, device="cuda")
    for r, n in enumerate(s["lens"].tolist()):
        lo = max(0, n - s["window"]) if s["window"] else 0
        blk = s["block_table"][r, :-(-n // bs)].long()

        def rows(cache, scale):
            x = cache[blk].double() * scale[blk].double()[:, :, None, None]
            return x.transpose(0, 1).reshape(Hkv, -1, D)[:, lo:n]

        score = rows(s["k_cache"], s["k_scale"]) @ s["q"][r].double().view(Hkv, G, D).transpose(1, 2).contiguous()
        score = score.transpose(1, 2).reshape(Hq, n - lo) * D ** -0.5
        every = score if s["sinks"] is None else torch.cat([score, s["sinks"].double()[:, None]], 1)
        lses[r] = torch.logsumexp(every, 1)
        p = torch.exp(score - lses[r][:, None]).view(Hkv, G, n - lo)
        out[r] = (p @ rows(s["v_cache"], s["v_scale"])).view(Hq, D)
    return out, lses


def _exact_copies(s):
    """Page by page, from copies of what the caches held."""
    bs, table = s["bs"], s["block_table"].tolist()
    moves = []  # page, its place, rows of it
    if s["op"] == "fork":
        lens = s["lens"].tolist()
        for p, page in zip(s["parent"].tolist(), s["page"].tolist()):
            if lens[p] % bs:
                moves.append((table[p][lens[p] // bs], page, lens[p] % bs))
    else:
        moves = [(b, to, bs) for b, to in enumerate(s["remap"].tolist()) if to >= 0 and to != b]
    after = []
    for which in ("k_cache", "v_cache", "k_scale", "v_scale"):
        x = s[which]
        if x is None or (s["kv"] == "int8" and which.endswith("cache")):
            if x is not None:
                after.append(None)  # codes: whole numbers, compared as they are
            continue
        y = x.clone() if s["kv"] != "fp8" else x.view(torch.uint8).clone().view(FP8)
        raw = torch.uint8 if s["kv"] == "fp8" else y.dtype
        for b, to, n in moves:
            if which.endswith("cache"):
                y.view(raw)[:, to, :, :n] = x.view(raw)[:, b, :, :n]
            else:
                y[:, to] = x[:, b]
        after.append(y.double())
    return (None, None, tuple(after)) if s["op"] == "fork" else (None, tuple(after))
