"""The attention calls reject bad arguments on the host, before anything is launched,
and the binding says which tensor is wrong (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2607_00466_amd import binding as B

P = ctypes.c_void_p(0x10000)    # 16-byte aligned, never dereferenced
ODD = ctypes.c_void_p(0x10002)  # aligned to nothing that the calls need
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return B.load()


def d(R=4, Hq=8, Hkv=2, D=128, bs=16, mb=8, nb=64, kv=torch.bfloat16, stride=0):
    return B.attn_dims(R, Hq, Hkv, D, bs, mb, nb, kv, stride)


def append(lib, dims=None, q=P, k=P, v=P, qs=1024, ks=256, vs=256, kind=0, T=3, pos=P, axes=1, axis=P, cos=P, sin=P,
           max_pos=64, rot=128, inter=0, slots=P, q_out=P, kc=P, vc=P):
    return lib.moe_kv_append(q, k, v, qs, ks, vs, kind, T, pos, axes, axis, cos, sin, max_pos, rot, inter, slots,
                             dims or d(), None, None, q_out, kc, vc, None)


def decode(lib, dims=None, q=P, k=P, v=P, table=P, lens=P, start=None, prefix=None, n=0, window=0, scale=0.1, out=P, lse=P, ws=P,
           ws_bytes=BIG, sinks=None):
    return lib.moe_attn_decode(q, k, v, table, lens, start, prefix, n, None, None, sinks, window, scale, dims or d(), out, lse, ws,
                               ws_bytes, None)


def weights(lib, dims=None, q=P, k=P, table=P, lens=P, start=None, prefix=None, n=0, scale=0.1, lse=P, w_in=P, w_out=P):
    return lib.moe_attn_weights(q, k, table, lens, start, prefix, n, None, scale, lse, dims or d(), w_in, w_out, None)


def evict(lib, dims=None, w=P, pos=P, lens=P, seen=P, protect=None, table=P, budget=16, recent=4, k=P, v=P, src=P,
          new=ctypes.c_void_p(0x20000), w_out=P, p_out=P):
    return lib.moe_kv_evict(w, pos, lens, seen, protect, table, dims or d(), budget, recent, k, v, src, new, w_out, p_out, None)


@pytest.mark.parametrize("dims,status", [
    (d(R=-1), B.MOE_ERR_INVALID),
    (d(Hq=7), B.MOE_ERR_INVALID),              # Hkv does not divide Hq
    (d(Hkv=0), B.MOE_ERR_INVALID),
    (d(bs=0), B.MOE_ERR_INVALID),
    (d(mb=-1), B.MOE_ERR_INVALID),
    (d(nb=-1), B.MOE_ERR_INVALID),
    (d(stride=2 * 16 * 128 - 16), B.MOE_ERR_INVALID),     # pages overlap
    (d(stride=2 * 16 * 128 + 8), B.MOE_ERR_UNSUPPORTED),  # rows off their alignment
    (d(R=1025), B.MOE_ERR_UNSUPPORTED),
    (d(Hq=512, Hkv=2), B.MOE_ERR_UNSUPPORTED),
    (d(D=96), B.MOE_ERR_UNSUPPORTED),
    (d(bs=8), B.MOE_ERR_UNSUPPORTED),
    (d(bs=24), B.MOE_ERR_UNSUPPORTED),
    (d(bs=2048), B.MOE_ERR_UNSUPPORTED),
    (d(mb=(1 << 15) + 1), B.MOE_ERR_UNSUPPORTED),         # 16 slots past the limit
])
def test_dims_rejected_by_every_call(lib, dims, status):
    assert append(lib, dims) == status
    assert decode(lib, dims) == status
    assert weights(lib, dims) == status
    assert evict(lib, dims) == status
    assert B.moe_attn_workspace_bytes(dims) == 0


def test_unknown_kv_type_rejected(lib):
    bad = d()
    bad.kv_type = 2
    for call in (append, decode, weights, evict):
        assert call(lib, bad) == B.MOE_ERR_INVALID
    with pytest.raises(ValueError, match="kv_dtype"):
        d(kv=torch.float16)


@pytest.mark.parametrize("args,status", [
    (dict(T=-1), B.MOE_ERR_INVALID),
    (dict(kind=2), B.MOE_ERR_INVALID),
    (dict(k=None), B.MOE_ERR_INVALID),
    (dict(v=None), B.MOE_ERR_INVALID),
    (dict(slots=None), B.MOE_ERR_INVALID),
    (dict(q=None), B.MOE_ERR_INVALID),           # q_out without q
    (dict(pos=None), B.MOE_ERR_INVALID),
    (dict(axis=None), B.MOE_ERR_INVALID),
    (dict(cos=None), B.MOE_ERR_INVALID),
    (dict(kc=None), B.MOE_ERR_INVALID),
    (dict(rot=-16), B.MOE_ERR_INVALID),
    (dict(rot=144), B.MOE_ERR_INVALID),          # more than D
    (dict(rot=24), B.MOE_ERR_UNSUPPORTED),
    (dict(ks=255), B.MOE_ERR_INVALID),           # rows overlap
    (dict(qs=1028), B.MOE_ERR_UNSUPPORTED),
    (dict(T=(1 << 20) + 1), B.MOE_ERR_UNSUPPORTED),
    (dict(axes=9), B.MOE_ERR_UNSUPPORTED),
    (dict(k=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(cos=ctypes.c_void_p(0x10004)), B.MOE_ERR_UNSUPPORTED),
    (dict(slots=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(T=0, k=None), B.MOE_OK),
])
def test_append_refusals(lib, args, status):
    assert append(lib, **args) == status


@pytest.mark.parametrize("args,status", [
    (dict(q=None), B.MOE_ERR_INVALID),
    (dict(k=None), B.MOE_ERR_INVALID),
    (dict(v=None), B.MOE_ERR_INVALID),
    (dict(table=None), B.MOE_ERR_INVALID),
    (dict(lens=None), B.MOE_ERR_INVALID),
    (dict(out=None), B.MOE_ERR_INVALID),
    (dict(ws=None), B.MOE_ERR_INVALID),
    (dict(n=1), B.MOE_ERR_INVALID),              # groups without their arrays
    (dict(n=-1), B.MOE_ERR_INVALID),
    (dict(n=1025, start=P, prefix=P), B.MOE_ERR_INVALID),
    (dict(window=-1), B.MOE_ERR_INVALID),
    (dict(scale=float("nan")), B.MOE_ERR_INVALID),
    (dict(q=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(out=ctypes.c_void_p(0x10008)), B.MOE_ERR_UNSUPPORTED),
    (dict(lens=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(lse=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(sinks=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(ws=ctypes.c_void_p(0x10004)), B.MOE_ERR_UNSUPPORTED),
    (dict(ws_bytes=1000), B.MOE_ERR_WORKSPACE),
    (dict(dims=d(R=0), q=None, lens=None), B.MOE_OK),
])
def test_decode_refusals(lib, args, status):
    assert decode(lib, **args) == status


@pytest.mark.parametrize("args,status", [
    (dict(q=None), B.MOE_ERR_INVALID),
    (dict(k=None), B.MOE_ERR_INVALID),
    (dict(lse=None), B.MOE_ERR_INVALID),
    (dict(w_out=None), B.MOE_ERR_INVALID),
    (dict(n=2), B.MOE_ERR_INVALID),
    (dict(scale=float("nan")), B.MOE_ERR_INVALID),
    (dict(w_out=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(lse=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(dims=d(R=0), q=None), B.MOE_OK),
    (dict(dims=d(nb=0), k=None), B.MOE_OK),
])
def test_weights_refusals(lib, args, status):
    assert weights(lib, **args) == status


@pytest.mark.parametrize("args,status", [
    (dict(budget=0), B.MOE_ERR_INVALID),
    (dict(recent=-1), B.MOE_ERR_INVALID),
    (dict(w=None), B.MOE_ERR_INVALID),
    (dict(pos=None), B.MOE_ERR_INVALID),
    (dict(lens=None), B.MOE_ERR_INVALID),
    (dict(seen=None), B.MOE_ERR_INVALID),
    (dict(src=None), B.MOE_ERR_INVALID),
    (dict(k=None), B.MOE_ERR_INVALID),
    (dict(new=P), B.MOE_ERR_INVALID),            # lens itself
    (dict(budget=(1 << 19) + 1), B.MOE_ERR_UNSUPPORTED),
    (dict(dims=d(R=1024, Hq=128, Hkv=128)), B.MOE_ERR_UNSUPPORTED),  # more rows than a grid has
    (dict(w=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(src=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(dims=d(R=0), w=None), B.MOE_OK),
])
def test_evict_refusals(lib, args, status):
    assert evict(lib, **args) == status


def test_limits_match_the_header():
    import os
    import re

    text = open(os.path.join(B.INCLUDE_DIR, "eldr_attention.h")).read()
    names = ["moe_kv_append", "moe_attn_workspace_bytes", "moe_attn_decode", "moe_attn_weights", "moe_kv_evict"]
    assert sorted(B.header_functions([os.path.join(B.INCLUDE_DIR, "eldr_attention.h")])) == sorted(names)
    assert set(names) <= set(B.header_functions())
    for name, value in (("MOE_KV_BF16", B.MOE_KV_BF16), ("MOE_KV_FP8", B.MOE_KV_FP8), ("MOE_IN_BF16", B.MOE_IN_BF16),
                        ("MOE_IN_FP32", B.MOE_IN_FP32)):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == value


def test_workspace_grows_with_the_rows(lib):
    small, large = B.moe_attn_workspace_bytes(d(R=1)), B.moe_attn_workspace_bytes(d(R=256))
    assert 0 < small < large
    # pages do not matter
    assert B.moe_attn_workspace_bytes(d(mb=1, nb=1)) == B.moe_attn_workspace_bytes(d(mb=999, nb=1 << 20))


def test_binding_names_the_tensor(lib):
    t = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q: must be a device tensor"):
        B.moe_attn_decode(t, t, t, t, t, d(), t, t, t)
    with pytest.raises(TypeError, match="q: expected a torch tensor"):
        B.moe_attn_weights(None, t, t, t, t, d(), t, t)
    with pytest.raises(ValueError, match="weights: must be a device tensor"):
        B.moe_kv_evict(t, t, t, t, t, d(), 16, 4, t, t, t, t, t, t)
    i = torch.zeros((1, 3), dtype=torch.int32)
    cs = torch.zeros((64, 64))
    with pytest.raises(ValueError, match="positions: expected"):
        B.moe_kv_append(t, t, t, i[:, :2], i, cs, cs, i, d(), t, t, t)
    with pytest.raises(ValueError, match="q and q_out come together"):
        B.moe_kv_append(t, t, t, i, i, cs, cs, i, d(), None, t, t)
    with pytest.raises(ValueError, match="come together"):
        B._need_groups(i, None)
