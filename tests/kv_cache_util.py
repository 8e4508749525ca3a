"""Inputs of the int8 cache's, the normed appends', forks' and compaction's GPU tests."""
from __future__ import annotations

import numpy as np
import torch

from paper_2607_00466_amd import binding as B

FP8 = torch.float8_e4m3fn
INT8 = torch.int8


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Rows:
    """T tokens' queries, keys and values (views of one projection's rows, heads of
    different size), rotation tables and norm weights, here and on the device."""

    def __init__(self, T, Hq, Hkv, D, rot, fp32=True, norms=True, axes=1, interleaved=False, seed=0, max_pos=97):
        rng = np.random.default_rng(seed)
        self.T, self.Hq, self.Hkv, self.D, self.interleaved = T, Hq, Hkv, D, interleaved
        heads = Hq + 2 * Hkv
        x = rng.standard_normal((T, heads, D)) * rng.uniform(0.05, 6.0, (1, heads, 1))
        qkv = torch.from_numpy(x.astype(np.float32)).cuda()
        qkv = qkv if fp32 else qkv.bfloat16()
        self.q, self.k, self.v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        angle = rng.uniform(-np.pi, np.pi, (max_pos, rot // 2))
        self.cos_np, self.sin_np = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
        self.positions_np = rng.integers(0, max_pos, (axes, T)).astype(np.int32)
        self.axis_np = rng.integers(0, axes, rot // 2).astype(np.int32)
        self.qn_np, self.kn_np = ((1 + 0.3 * rng.standard_normal(D)).astype(np.float32) if norms else None for _ in "qk")
        self.cos, self.sin, self.positions, self.axis = dev(self.cos_np), dev(self.sin_np), dev(self.positions_np), dev(self.axis_np)
        self.q_norm, self.k_norm = (None if w is None else dev(w) for w in (self.qn_np, self.kn_np))
        self.q_out = torch.full((T, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")

    def numpy(self, which):
        return getattr(self, which).float().cpu().numpy()

    def expected(self, which, eps=1e-6, exact=False):
        """Queries or keys as they are rounded for q_out or the cache: fp32, or 64 bits."""
        from oracle import kv_cache as K

        x = K.normed(self.numpy(which), self.qn_np if which == "q" else self.kn_np, eps, exact)
        return K.turned(x, self.positions_np, self.axis_np, self.cos_np, self.sin_np, self.interleaved)


class Int8Cache:
    """An int8 cache whose pages and scales hold anything before."""

    def __init__(self, nb, Hkv, bs, D, seed=0, pad=0):
        rng = np.random.default_rng(seed)
        self.nb, self.Hkv, self.bs, self.D = nb, Hkv, bs, D
        self.stride = Hkv * bs * D + pad
        self.block_stride = self.stride if pad else 0
        self.k, self.v = (self._place(rng.integers(-127, 128, (nb, Hkv, bs, D)).astype(np.int8)) for _ in "kv")
        self.k_scale, self.v_scale = (dev(rng.uniform(0.001, 0.05, (nb, Hkv)).astype(np.float32)) for _ in "kv")

    def _place(self, x):
        buf = torch.zeros(self.nb * self.stride, dtype=INT8, device="cuda")
        t = torch.as_strided(buf, x.shape, (self.stride, self.bs * self.D, self.D, 1))
        t.copy_(torch.from_numpy(x))
        return t

    def dims(self, R, Hq, max_blocks):
        return B.attn_dims(R, Hq, self.Hkv, self.D, self.bs, max_blocks, self.nb, INT8, self.block_stride)

    def numpy(self):
        return self.k.cpu().numpy(), self.k_scale.cpu().numpy(), self.v.cpu().numpy(), self.v_scale.cpu().numpy()


def append_int8(rows, cache, query_start, table, lens, q=True, eps=1e-6, stream=None):
    table = np.asarray(table, np.int32)
    B.moe_kv_append_int8(rows.q if q else None, rows.k, rows.v, rows.positions, rows.axis, rows.cos, rows.sin, i32(query_start),
                         i32(table), i32(lens), cache.dims(len(lens), rows.Hq, table.shape[1]), rows.q_out if q else None, cache.k,
                         cache.v, cache.k_scale, cache.v_scale, q_norm=rows.q_norm, k_norm=rows.k_norm, eps=eps,
                         interleaved=rows.interleaved, stream=stream)


def check_append_int8(rows, cache, before, query_start, table, lens, eps=1e-6):
    """The caches, bit for bit, against the oracle's from what they held before."""
    from oracle import kv_cache as K

    torch.cuda.synchronize()
    k0, ks0, v0, vs0 = before
    k1, ks1, v1, vs1 = cache.numpy()
    for got, got_scale, x, was, was_scale, name in ((k1, ks1, rows.expected("k", eps), k0, ks0, "keys"),
                                                    (v1, vs1, rows.numpy("v"), v0, vs0, "values")):
        want, scale = K.append_int8(x, query_start, table, lens, was, was_scale)
        np.testing.assert_array_equal(got_scale, scale, err_msg=name + "' scales")
        np.testing.assert_array_equal(got, want, err_msg=name)


def bits(t):
    return t.contiguous().view(torch.uint8 if t.element_size() == 1 else torch.int16 if t.element_size() == 2 else torch.int32)
