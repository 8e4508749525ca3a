"""The calls of eldr_kv_cache.h, and the attention calls on a cache of 8-bit integers,
reject bad arguments on the host, before anything is launched (no GPU needed)."""
import ctypes
import os
import re

import pytest
import torch

from paper_2607_00466_amd import binding as B

P = ctypes.c_void_p(0x10000)    # 16-byte aligned, never dereferenced
ODD = ctypes.c_void_p(0x10002)  # aligned to nothing that the calls need
FOUR = ctypes.c_void_p(0x10004)
BIG = 1 << 40
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return B.load()


def d(R=4, Hq=8, Hkv=2, D=128, bs=16, mb=8, nb=64, kv=torch.int8, stride=0):
    return B.attn_dims(R, Hq, Hkv, D, bs, mb, nb, kv, stride)


def norm(lib, dims=None, q=P, k=P, v=P, qs=1024, ks=256, vs=256, kind=0, T=3, pos=P, axes=1, axis=P, cos=P, sin=P, max_pos=64,
         rot=128, inter=0, slots=P, qn=P, kn=P, eps=1e-6, k_scale=None, v_scale=None, q_out=P, kc=P, vc=P):
    return lib.moe_kv_append_norm(q, k, v, qs, ks, vs, kind, T, pos, axes, axis, cos, sin, max_pos, rot, inter, slots,
                                  dims or d(kv=torch.bfloat16), qn, kn, eps, k_scale, v_scale, q_out, kc, vc, None)


def int8(lib, dims=None, q=P, k=P, v=P, qs=1024, ks=256, vs=256, kind=0, T=3, pos=P, axes=1, axis=P, cos=P, sin=P, max_pos=64,
         rot=128, inter=0, start=P, table=P, lens=P, qn=P, kn=P, eps=1e-6, q_out=P, kc=P, vc=P, k_scale=P, v_scale=P):
    return lib.moe_kv_append_int8(q, k, v, qs, ks, vs, kind, T, pos, axes, axis, cos, sin, max_pos, rot, inter, start, table, lens,
                                  dims or d(), qn, kn, eps, q_out, kc, vc, k_scale, v_scale, None)


def fork(lib, dims=None, parent=P, child=P, page=P, F=2, table=P, lens=P, layers=3, stride=0, kc=P, vc=P, k_scale=P, v_scale=P):
    return lib.moe_kv_fork(parent, child, page, F, table, lens, dims or d(), layers, stride, kc, vc, k_scale, v_scale, None)


def compact(lib, dims=None, remap=P, table=P, out=P, layers=3, stride=0, kc=P, vc=P, k_scale=P, v_scale=P):
    return lib.moe_kv_compact(remap, table, out, dims or d(), layers, stride, kc, vc, k_scale, v_scale, None)


CALLS = [norm, int8, fork, compact]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("change,status", [
    (dict(R=-1), B.MOE_ERR_INVALID), (dict(Hq=7), B.MOE_ERR_INVALID), (dict(bs=0), B.MOE_ERR_INVALID),
    (dict(stride=2 * 16 * 128 - 16), B.MOE_ERR_INVALID), (dict(stride=2 * 16 * 128 + 8), B.MOE_ERR_UNSUPPORTED),
    (dict(R=1025), B.MOE_ERR_UNSUPPORTED), (dict(D=96), B.MOE_ERR_UNSUPPORTED), (dict(bs=24), B.MOE_ERR_UNSUPPORTED),
    (dict(mb=(1 << 15) + 1), B.MOE_ERR_UNSUPPORTED)])
def test_dims_rejected_by_every_call(lib, call, change, status):
    assert call(lib, d(kv=torch.bfloat16 if call is norm else torch.int8, **change)) == status


APPENDS = [
    (dict(T=-1), B.MOE_ERR_INVALID),
    (dict(kind=2), B.MOE_ERR_INVALID),
    (dict(k=None), B.MOE_ERR_INVALID),
    (dict(v=None), B.MOE_ERR_INVALID),
    (dict(q=None), B.MOE_ERR_INVALID),           # q_out without q
    (dict(pos=None), B.MOE_ERR_INVALID),
    (dict(cos=None), B.MOE_ERR_INVALID),
    (dict(kc=None), B.MOE_ERR_INVALID),
    (dict(rot=144), B.MOE_ERR_INVALID),          # more than D
    (dict(rot=24), B.MOE_ERR_UNSUPPORTED),
    (dict(ks=255), B.MOE_ERR_INVALID),           # rows overlap
    (dict(qs=1028), B.MOE_ERR_UNSUPPORTED),
    (dict(T=(1 << 20) + 1), B.MOE_ERR_UNSUPPORTED),
    (dict(axes=9), B.MOE_ERR_UNSUPPORTED),
    (dict(k=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(cos=FOUR), B.MOE_ERR_UNSUPPORTED),
    (dict(eps=-1e-9), B.MOE_ERR_INVALID),
    (dict(eps=NAN), B.MOE_ERR_INVALID),
    (dict(eps=INF), B.MOE_ERR_INVALID),
    (dict(qn=FOUR), B.MOE_ERR_UNSUPPORTED),
    (dict(kn=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(T=0, k=None), B.MOE_OK),
]


@pytest.mark.parametrize("args,status", APPENDS + [
    (dict(slots=None), B.MOE_ERR_INVALID),
    (dict(slots=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(k_scale=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(dims=d()), B.MOE_ERR_UNSUPPORTED),     # a cache of 8-bit integers
])
def test_append_norm_refusals(lib, args, status):
    assert norm(lib, **args) == status


@pytest.mark.parametrize("args,status", APPENDS + [
    (dict(start=None), B.MOE_ERR_INVALID),
    (dict(table=None), B.MOE_ERR_INVALID),
    (dict(lens=None), B.MOE_ERR_INVALID),
    (dict(k_scale=None), B.MOE_ERR_INVALID),
    (dict(v_scale=None), B.MOE_ERR_INVALID),
    (dict(start=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(lens=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(v_scale=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(dims=d(kv=torch.bfloat16)), B.MOE_ERR_INVALID),
    (dict(dims=d(kv=torch.float8_e4m3fn)), B.MOE_ERR_INVALID),
    (dict(dims=d(R=0), start=None), B.MOE_OK),
])
def test_append_int8_refusals(lib, args, status):
    assert int8(lib, **args) == status


@pytest.mark.parametrize("args,status", [
    (dict(F=-1), B.MOE_ERR_INVALID),
    (dict(F=65536), B.MOE_ERR_UNSUPPORTED),
    (dict(parent=None), B.MOE_ERR_INVALID),
    (dict(child=None), B.MOE_ERR_INVALID),
    (dict(page=None), B.MOE_ERR_INVALID),
    (dict(table=None), B.MOE_ERR_INVALID),
    (dict(lens=None), B.MOE_ERR_INVALID),
    (dict(page=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(F=0, parent=None), B.MOE_OK),
    (dict(dims=d(R=0), parent=None), B.MOE_OK),
])
def test_fork_refusals(lib, args, status):
    assert fork(lib, **args) == status


@pytest.mark.parametrize("args,status", [
    (dict(remap=None), B.MOE_ERR_INVALID),
    (dict(table=None), B.MOE_ERR_INVALID),
    (dict(out=None), B.MOE_ERR_INVALID),
    (dict(remap=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(out=ODD), B.MOE_ERR_UNSUPPORTED),
    (dict(dims=d(R=0, nb=0), remap=None, kc=None, vc=None), B.MOE_OK),
])
def test_compact_refusals(lib, args, status):
    assert compact(lib, **args) == status


@pytest.mark.parametrize("call", [fork, compact])
@pytest.mark.parametrize("args,status", [
    (dict(layers=-1), B.MOE_ERR_INVALID),
    (dict(layers=1025), B.MOE_ERR_UNSUPPORTED),
    (dict(stride=-16), B.MOE_ERR_INVALID),
    (dict(stride=64 * 4096 + 8), B.MOE_ERR_UNSUPPORTED),
    (dict(stride=64 * 4096 - 16), B.MOE_ERR_INVALID),                          # layers overlap
    (dict(stride=4096, dims=d(stride=2 * 4096)), B.MOE_ERR_INVALID),           # two layers fit beside each other, not three
    (dict(stride=4096 - 16, dims=d(stride=4 * 4096)), B.MOE_ERR_INVALID),
    (dict(kc=None), B.MOE_ERR_INVALID),
    (dict(vc=None), B.MOE_ERR_INVALID),
    (dict(k_scale=None), B.MOE_ERR_INVALID),
    (dict(v_scale=None), B.MOE_ERR_INVALID),
    (dict(kc=FOUR), B.MOE_ERR_UNSUPPORTED),
    (dict(k_scale=ODD), B.MOE_ERR_UNSUPPORTED),
])
def test_layers_refusals(lib, call, args, status):
    assert call(lib, **args) == status


def test_attention_on_8_bit_integers(lib):
    def decode(k_scale=P, v_scale=P, dims=None):
        return lib.moe_attn_decode(P, P, P, P, P, None, None, 0, k_scale, v_scale, None, 0, 0.1, dims or d(), P, P, P, 0, None)

    assert decode(k_scale=None) == decode(v_scale=None) == B.MOE_ERR_INVALID  # its scales are not optional
    assert decode(k_scale=ODD) == B.MOE_ERR_UNSUPPORTED
    assert decode() == B.MOE_ERR_WORKSPACE
    assert B.moe_attn_workspace_bytes(d()) == B.moe_attn_workspace_bytes(d(kv=torch.bfloat16))
    # what knows no pages' scales
    assert lib.moe_kv_append(P, P, P, 1024, 256, 256, 0, 3, P, 1, P, P, P, 64, 128, 0, P, d(), None, None, P, P, P, None) == B.MOE_ERR_UNSUPPORTED
    assert lib.moe_attn_weights(P, P, P, P, None, None, 0, None, 0.1, P, d(), P, P, None) == B.MOE_ERR_UNSUPPORTED
    assert lib.moe_kv_evict(P, P, P, P, None, P, d(), 16, 4, P, P, P, ctypes.c_void_p(0x20000), P, P, None) == B.MOE_ERR_UNSUPPORTED


def test_limits_match_the_header():
    path = os.path.join(B.INCLUDE_DIR, "eldr_kv_cache.h")
    names = ["moe_kv_append_norm", "moe_kv_append_int8", "moe_kv_fork", "moe_kv_compact"]
    assert sorted(B.header_functions([path])) == sorted(names) and set(names) <= set(B.header_functions())
    text = open(os.path.join(B.INCLUDE_DIR, "eldr_attention.h")).read()
    assert int(re.search(r"#define MOE_KV_INT8 (\d+)", text).group(1)) == B.MOE_KV_INT8


def test_binding_names_the_tensor(lib):
    t = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    i = torch.zeros((1, 4), dtype=torch.int32)
    cs, axis = torch.zeros((64, 64)), torch.zeros(64, dtype=torch.int32)
    with pytest.raises(ValueError, match="positions: expected"):
        B.moe_kv_append_norm(t, t, t, i[:, :2], axis, cs, cs, i, d(kv=torch.bfloat16), t, t, t, None, None)
    with pytest.raises(ValueError, match="q and q_out come together"):
        B.moe_kv_append_int8(t, t, t, i, axis, cs, cs, i, i, i, d(), None, t, t, t, t)
    with pytest.raises(ValueError, match="q: must be a device tensor"):
        B.moe_kv_append_int8(t, t, t, i, axis, cs, cs, i, i, i, d(), t, t, t, t, t)
    with pytest.raises(ValueError, match="parent: must be a device tensor"):
        B.moe_kv_fork(i, i, i, i, i, d(), t, t)
    with pytest.raises(ValueError, match="remap: must be a device tensor"):
        B.moe_kv_compact(i, i, i, d(), t, t)
    with pytest.raises(ValueError, match=r"k_cache: expected \[num_blocks"):
        B._need_layers(t, t, None, None, d())
    with pytest.raises(ValueError, match="k_scale and v_scale: a cache of torch.int8 has both"):
        B._need_scales(None, t, d())


def test_the_example_evicts_nothing_of_8_bit_integers():
    from examples import decode_step as E
    from paper_2607_00466_amd import synth

    for bad in (dict(budget=50), dict(fp8=True)):
        sizes = dict(R=4, groups=2, prefix=32, own=16, budget=64, steps=3, recent=4, int8=True) | bad
        with pytest.raises(ValueError, match="8-bit integers"):
            E.Worker(synth.SHAPES["tiny"], E.Heads(4, 2, 64), **sizes)


@pytest.mark.parametrize("kv", [torch.bfloat16, torch.int8])
def test_layers_that_are_one(lib, kv):
    """An expanded cache has a layer stride of 0, which the library takes for dense layers
    and would write past the one that is there."""
    dims = d(kv=kv)
    whole = torch.zeros((3, 64, 2, 16, 128), dtype=kv)
    one = whole[:1].expand(3, -1, -1, -1, -1)
    for k, v, name in ((one, one, "k_cache"), (one, whole, "k_cache")):
        with pytest.raises(ValueError, match=f"{name}: an expanded tensor's layers are all the same one"):
            B._need_layers(k, v, None, None, dims)
    with pytest.raises(ValueError, match="must be a device tensor"):  # (one layer, expanded or not, has no stride)
        B._need_layers(whole[:1].expand(1, -1, -1, -1, -1), whole[:1], None, None, dims)
