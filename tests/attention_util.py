"""Inputs and comparisons of the attention calls' GPU tests."""
from __future__ import annotations

import numpy as np
import torch

from oracle import attention as A
from paper_2607_00466_amd import binding as B

FP8 = torch.float8_e4m3fn

# Unit roundoffs: to bf16 (8 significant bits), to e4m3 (4), to fp32 (24).
U_BF16, U_FP8, U_FP32 = 2.0 ** -8, 2.0 ** -4, 2.0 ** -24


class Cache:
    """Random keys and values in scattered pages, every slot that no request has
    cached (and every page that no table names) holding NaN or infinities."""

    def __init__(self, lens, Hkv, D, bs, fp8=False, seed=0, shared=(), max_blocks=None, spare=3, pad=0, amp=1.0):
        """shared: (first request, end, tokens) of each group; the members' own pages
        start after the shared ones, and their table entries before are -1."""
        rng = np.random.default_rng(seed)
        R = len(lens)
        want = [max(0, -(-n // bs)) for n in lens]
        self.max_blocks = max_blocks or max([1] + want)
        ids = list(rng.permutation(sum(want) + spare))
        self.nb = len(ids)
        table = np.full((R, self.max_blocks), -1, np.int32)
        for r in range(R):
            skip = 0
            for s, e, tokens in shared:
                if s < r < e:
                    skip = min(tokens // bs, want[r])
            for i in range(skip, want[r]):
                table[r, i] = ids.pop()
            for s, e, tokens in shared:
                # a page that the prefix ends inside holds its shared tokens in every member's copy too
                if s < r < e and tokens % bs and tokens // bs < want[r]:
                    self.copies = getattr(self, "copies", []) + [(table[s, tokens // bs], table[r, tokens // bs], tokens % bs)]
        self.table_np, self.lens_np, self.bs, self.D, self.Hkv, self.fp8 = table, np.array(lens), bs, D, Hkv, fp8
        self.N = self.max_blocks * bs
        garbage = np.array([np.nan, np.inf, -np.inf, 3e38], np.float32)
        stored = []
        for which in range(2):
            x = (rng.standard_normal((self.nb, Hkv, bs, D)) * amp).astype(np.float32)
            used = np.zeros((self.nb, bs), bool)
            for r in range(R):
                for j in range(min(lens[r], self.N)):
                    if table[r, j // bs] >= 0:
                        used[table[r, j // bs], j % bs] = True
            for a, b, n in getattr(self, "copies", []):
                x[b, :, :n] = x[a, :, :n]
            bad = ~np.broadcast_to(used[:, None, :, None], x.shape)
            x[bad] = garbage[rng.integers(0, 4, int(bad.sum()))]
            stored.append(torch.from_numpy(x))
        dtype = FP8 if fp8 else torch.bfloat16
        stride = Hkv * bs * D + pad
        self.block_stride = stride if pad else 0
        self.k, self.v = (self._place(x.to(dtype), stride) for x in stored)
        self.k_scale = self.v_scale = None
        ks = vs = np.ones(Hkv)
        if fp8:
            ks, vs = rng.uniform(0.5, 1.5, (2, Hkv)).astype(np.float32)
            self.k_scale, self.v_scale = torch.from_numpy(ks).cuda(), torch.from_numpy(vs).cuda()
        # what the caches stand for, in 64 bits
        self.k_np = self.k.cpu().double().numpy() * ks.astype(np.float64)[:, None, None]
        self.v_np = self.v.cpu().double().numpy() * vs.astype(np.float64)[:, None, None]
        self.table, self.lens = torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")

    @staticmethod
    def _place(x, stride):
        nb, Hkv, bs, D = x.shape
        buf = torch.zeros(nb * stride, dtype=x.dtype, device="cuda")
        t = torch.as_strided(buf, (nb, Hkv, bs, D), (stride, bs * D, D, 1))
        t.copy_(x.cuda())
        return t

    def dims(self, Hq):
        return B.attn_dims(len(self.lens_np), Hq, self.Hkv, self.D, self.bs, self.max_blocks, self.nb,
                           FP8 if self.fp8 else torch.bfloat16, self.block_stride)


def groups_of(shared, R):
    """group_start and prefix_len (device, host) of [(first, end, tokens)], ascending."""
    if not shared:
        return None, None, None, None
    start, prefix, at = [], [], 0
    for s, e, tokens in shared:
        if s > at or not start:
            if s > at:
                start.append(at)
                prefix.append(0)
        start.append(s)
        prefix.append(tokens)
        at = e
    start.append(at)
    t = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return t(start), t(prefix), start, prefix


def queries(R, Hq, D, seed=0, amp=1.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((R, Hq, D), generator=g) * amp).to(torch.bfloat16).cuda()


def score_bound(q, cache, scale):
    """A bound on the fp32 error of any score: the products' sum of D + 8 roundings
    (and the scale's) over the largest sum of absolute products."""
    k = np.abs(cache.k_np)
    k = np.where(np.isfinite(k) & (k < 1e30), k, 0)
    biggest = np.linalg.norm(q.double().cpu().numpy(), axis=-1).max() * np.linalg.norm(k, axis=-1).max() * abs(scale)
    return (cache.D + 8) * U_FP32 * biggest


def check_decode(out, lse, q, cache, scale, ref, sinks=None):
    """out and lse against the oracle's (out, lse, mass).

    With e the scores' error, a weight is off by a factor within 2 e + a few fp32
    roundings (its own score and lse) and by its rounding to bf16; out then by that
    much of mass = sum p |v|, and by its own rounding to bf16.  lse is off by e and
    fp32 roundings of its own value and of the logarithm's."""
    want, want_lse, mass = ref
    e = score_bound(q, cache, scale)
    rel = np.expm1(2 * e) + 64 * U_FP32
    got = out.double().cpu().numpy()
    tol = (U_BF16 + rel) * mass * 1.01 + U_BF16 * 1.01 * np.abs(want) + 1e-38
    off = np.abs(got - want)
    assert np.isfinite(got).all()
    assert (off <= tol).all(), f"out off by {(off / np.maximum(tol, 1e-300)).max():.3g} of its bound"
    if lse is not None:
        got = lse.double().cpu().numpy()
        empty = np.isinf(want_lse)
        assert np.array_equal(np.isinf(got), empty) and (got[empty] < 0).all()
        off = np.abs(got[~empty] - want_lse[~empty])
        tol = e + 16 * U_FP32 * (1 + np.abs(want_lse[~empty]))
        assert (off <= tol).all(), f"lse off by {(off / tol).max():.3g} of its bound"


def run_decode(cache, q, shared=(), sinks=None, window=0, scale=None, ws=None, check=True, stream=None):
    R, Hq, D = q.shape
    d = cache.dims(Hq)
    gs, pl, gs_np, pl_np = groups_of(shared, R)
    out = torch.full((R, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((R, Hq), float("nan"), device="cuda")
    if ws is None:
        ws = B.attn_workspace(d)
        ws.fill_(float("nan"))  # its contents mean nothing
    B.moe_attn_decode(q, cache.k, cache.v, cache.table, cache.lens, d, out, lse, ws, gs, pl, cache.k_scale,
                      cache.v_scale, sinks, window, scale, stream=stream)
    torch.cuda.synchronize()
    if check:
        s = D ** -0.5 if scale is None else scale
        ref = A.decode(q.double().cpu().numpy(), cache.k_np, cache.v_np, cache.table_np, cache.lens_np, s, gs_np, pl_np,
                       None if sinks is None else sinks.double().cpu().numpy(), window)
        check_decode(out, lse, q, cache, s, ref)
    return out, lse
